// Causal differential attention of new tokens over the 8-bit paged K/V cache (include/hgf.h, hgf_diff_attention_cached).
//
// What a page's head costs to read is 3 * 64 * DH bytes, and for few query rows every byte is used for few products: a stream from memory.  The work is
// cut into units of that size - a page of a sequence and K/V head, or 32 open tokens - and the units of all (sequence, group of query rows, head)
// items are laid in one sequence, which is dealt in equal shares to one CTA an SM and within a CTA to its teams of warps.  A team has a ring of
// units in shared memory that bulk copies fill, and works alone.  An item that lies within one team's share is finished there; of an item that
// several share each leaves its softmax statistics and sums in the workspace.  What teams of one CTA share is joined at the end of that CTA, what
// several CTAs share by a second kernel, both in the order of the tokens: the same call gives the same bits.
//
// Products are int8 tensor-core products on the codes as they lie in the page (m16n8k32, the codes as left operand), exact:
//   scores   q as a 23-bit fixed-point number of the row's power of two, cut into three signed digits in base 256: columns of the right operand
//   values   probabilities relative to the largest of the row's in this page, as fixed-point numbers of 24 bits (the bits of 1 + p), three unsigned
//            digits, whatever the output's type (two digits, 16 bits, moved one bf16 output in a hundred to its neighbour for 3 us of the 55 below)
// The accumulators start at the bits of 1.5 * 2^23, so that a sum, below 2^22 in magnitude, is a float after one subtraction: I2F runs at an eighth
// of the FMA rate and bounded the kernel.  The open tokens' bf16 go through bf16 products, with the probabilities as sums of three bf16.
//
// Four forms.  Many rows are tcgen05 products (hgf_cached_attention_tc.cuh).  Here ROWS = 1, for single tokens with heads of their own: a warp is a team, both streams' digits fit the eight columns of one product.  There
// and with ROWS = 8, a few tokens or heads that share K and V, the codes are the left operand, tokens (or dims) as its rows; eight query rows are the
// columns of a product for each digit, and a team is a warp for each stream.  ROWS = 16, for more: sixteen query rows are the left operand and the
// codes the right one (a lane's sixteen bytes are the same either way round); a warp takes one stream of one tile of sixteen rows, and a team is the
// warps of one or two tiles, so that a page that is read once serves up to 32 rows.  There the columns of the scores' products are the page's tokens in
// such an order that a lane gets four neighbouring tokens of its rows: the probabilities' digits are then in place for the second product, where
// ROWS = 8 turns the scores through shared memory.
//
// Measured (one B200; floor: the cache's bytes once at 6567 GB/s of copy bandwidth):
//   single tokens   64 sequences of up to 4096 tokens, 16 heads of 128: 248 us, 99 % of the floor's rate; one of 131071 tokens, 16 heads of 64: 73 us, 84 %;
//                   32 of up to 2048: 32 us, 63 % - 4 us to begin, unequal ends of the CTAs, the join; one of 200 tokens: 9 us, launches and look-ups
//   shared heads    16 sequences of up to 2900 tokens, 5 drafts of 4 query heads a K/V head, 128 wide: 55 us, floor 14.  Bound by dependent issue at two warps
//                   a scheduler (0.30 instructions issued a clock; 1600 a page, stream and sixteen rows with waits and items' ends, 192 of them products; integer tensor
//                   pipe 28 % busy).  Most sequences have one tile of sixteen, three of the sixteen two: 63 % of the tiles' rows are there.
//                   Tiles of eight rows against sixteen: one sequence of 59361 tokens, two heads a K/V head, 128 wide 71 and 110 us; with sixteen warps instead of
//                   eight for those, 64 wide, 51 and 49 (13 sequences of 5 tokens 13.6 and 9.9)
#include "hgf_cache.cuh"
#include "hgf_warp.cuh"

namespace hgf {

constexpr int kCaMaxSms = 160;      // CTAs at most (the workspace has room for them)
constexpr int kCaMaxTeams = 8;      // teams of a CTA at most

template <int DH, int ROWS>
struct CaCfg {
    static constexpr int WARPS = ROWS == 1 && DH == 128 ? 4 : 8, THREADS = WARPS * 32;
    static constexpr int UNIT = 3 * kCacheBlock * DH;            // bytes of a unit
    static constexpr int STAGE = (UNIT + 16 + 127) / 128 * 128;  // with the page's scales
    static constexpr int STAGES = DH == 64 ? 16 : 8;             // of all teams' rings
    static constexpr int KT = DH / 32, MT = DH / 16;
    static constexpr int SCORES = ROWS == 1 ? 2 * kCacheBlock * 4 : ROWS == 8 ? 8 * 36 * 4 : 0;  // bytes a warp; rows 36 floats apart: eight rows' writes hit all banks
    static constexpr int PART = 4 + 2 * DH;                      // floats: maximum and sum of stream 1, of stream 2, sums of values of both
    // (prefix sums, rounded up to 16 bytes; of single tokens the parts, two a warp; of sixteen rows room for 64 dims of the second stream's sums, for each
    // pair of warps, in rows 68 floats apart, which with eight rows is the pair's room for scores)
    static constexpr int PREFIX = (kCacheMaxSeqs + 2) * 8, GIVEN = 16 * 68, PARTS = ROWS == 1 ? WARPS * 2 * PART * 4 : ROWS == 16 ? WARPS / 2 * GIVEN * 4 : 0;
    static constexpr int SMEM = STAGES * STAGE + WARPS * SCORES + PREFIX + PARTS;
};

struct CaParams {
    CacheView c;
    const __nv_bfloat16 *q;
    const int32_t *slots, *starts;
    void *out;
    int4 *items;          // [CTAs][2]: what the joining kernel does for a CTA
    float *cta_parts;     // [CTAs][2][tiles][ROWS][PART]
    float *parts;         // [CTAs][teams][2][tiles][ROWS][PART], ROWS > 1
    unsigned int *status;
    int n_seqs, n_rows, group, bf16;
    int teams, tiles, stages;  // of a CTA; of a team; of a team's ring
    float lambda, out_scale, scale_log2, per_group;  // (per_group: 1 / group)
};

// d = c + a b; c may be d.
__device__ __forceinline__ void mma_s8s8(int (&d)[4], const uint4 &a, uint32_t b0, uint32_t b1, const int (&c)[4]) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};\n"
                 : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
                 : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1), "r"(c[0]), "r"(c[1]), "r"(c[2]), "r"(c[3]));
}
__device__ __forceinline__ void mma_s8u8(int (&d)[4], const uint4 &a, uint32_t b0, uint32_t b1, const int (&c)[4]) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.u8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};\n"
                 : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
                 : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1), "r"(c[0]), "r"(c[1]), "r"(c[2]), "r"(c[3]));
}
__device__ __forceinline__ void mma_u8s8(int (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, const int (&c)[4]) {
    asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};\n"
                 : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "r"(c[0]), "r"(c[1]), "r"(c[2]), "r"(c[3]));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint4 &a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
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


constexpr uint32_t kCaMagic = 0x4b400000u;      // 1.5 * 2^23: an accumulator that starts there is that float plus its sum
constexpr float kCaMagicF = 12582912.0f;
__device__ __forceinline__ float ca_float(int d) { return __int_as_float(d) - kCaMagicF; }
__device__ __forceinline__ uint64_t ca_float2(int a, int b) {
    return add_f32x2(pack_f32x2(__int_as_float(a), __int_as_float(b)), pack_f32x2(-kCaMagicF, -kCaMagicF));
}

// A sequence of the call; its items are tiles tile0 .. tiles - 1, since no row of those before sees a token.
struct CaSeq {
    int slot, row0, m, length, pages, units, tile0, tiles;
};
__device__ __forceinline__ CaSeq ca_sequence(const CaParams &p, int rows, int i) {
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
    // (one more for what an item costs apart from its units, to begin and to end: no token is in it, so nothing is read)
    s.units = s.length ? s.pages + (open > 0) + (open > 32) + 1 : 0;
    s.tiles = (s.m * p.group + rows - 1) / rows;
    s.tile0 = s.m > s.length ? (s.m - s.length) * p.group / rows : 0;
    return s;
}
// total * i / n and its inverse, the share of n that `unit` is in; i and n at most 1024 (a 64-bit division takes some 150 clocks, a 32-bit one 30).
__device__ __forceinline__ long long ca_share(long long total, int i, int n) {
    return total < (1 << 21) ? (long long)((uint32_t)total * (uint32_t)i / (uint32_t)n) : total * i / n;
}
__device__ __forceinline__ int ca_share_of(long long total, long long unit, int n) {
    return total < (1 << 21) ? (int)((((uint32_t)unit + 1) * (uint32_t)n - 1) / (uint32_t)total) : (int)(((unit + 1) * n - 1) / total);
}
// A unit's place: its sequence, the item's rows and head, its number in the item.
struct CaCursor {
    CaSeq s;
    int seq, tile, head, unit;
};
// An item as it is left for joining: its first unit and the one behind its last, and where its rows go.
struct CaItem {
    long long from, to;
    int row0, m, head, tile;
};

__device__ __forceinline__ void ca_write(const CaParams &p, const CaItem &it, int rr, int dh, int dim, float y) {
    const size_t o = ((size_t)(it.row0 + rr / p.group) * p.c.H * p.group + it.head * p.group + rr % p.group) * dh + dim;
    if (p.bf16) reinterpret_cast<__nv_bfloat16 *>(p.out)[o] = __float2bfloat16(y);
    else reinterpret_cast<float *>(p.out)[o] = y;
}

__device__ __forceinline__ void ca_put2(const CaParams &p, size_t at, float y0, float y1) {
    if (p.bf16) *reinterpret_cast<__nv_bfloat162 *>(reinterpret_cast<__nv_bfloat16 *>(p.out) + at) = __floats2bfloat162_rn(y0, y1);
    else *reinterpret_cast<float2 *>(reinterpret_cast<float *>(p.out) + at) = make_float2(y0, y1);
}
__device__ __forceinline__ void ca_write2(const CaParams &p, const CaItem &it, int rr, int dh, int dim, float y0, float y1) {
    ca_put2(p, ((size_t)(it.row0 + rr / p.group) * p.c.H * p.group + it.head * p.group + rr % p.group) * dh + dim, y0, y1);
}

// What parts of an item add up to, for four dims of a row.
struct CaSum {
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {}, o[2][4] = {};

    __device__ __forceinline__ void add(const float4 &ml, const float4 &v1, const float4 &v2) {
        const float pm[2] = {ml.x, ml.z}, pl[2] = {ml.y, ml.w}, v[2][4] = {{v1.x, v1.y, v1.z, v1.w}, {v2.x, v2.y, v2.z, v2.w}};
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const float now = fmaxf(m[s], pm[s]), base = now == -INFINITY ? 0.0f : now, a = exp2_approx(m[s] - base), c = exp2_approx(pm[s] - base);
            l[s] = l[s] * a + pl[s] * c;
#pragma unroll
            for (int d = 0; d < 4; ++d) o[s][d] = o[s][d] * a + v[s][d] * c;
            m[s] = now;
        }
    }
    __device__ __forceinline__ void add_part(const float *part, int dh, int dim, int fours = 1) {  // (each four floats of a part `fours` of such from the last)
        const float4 *at = reinterpret_cast<const float4 *>(part);
        add(*at, at[(1 + (dim >> 2)) * fours], at[(1 + ((dh + dim) >> 2)) * fours]);
    }
    __device__ __forceinline__ void store_part(float *part, int dh, int dim, bool first) const {
        if (first) *reinterpret_cast<float4 *>(part) = make_float4(m[0], l[0], m[1], l[1]);
        *reinterpret_cast<float4 *>(part + 4 + dim) = make_float4(o[0][0], o[0][1], o[0][2], o[0][3]);
        *reinterpret_cast<float4 *>(part + 4 + dh + dim) = make_float4(o[1][0], o[1][1], o[1][2], o[1][3]);
    }
    __device__ __forceinline__ void write(const CaParams &p, const CaItem &it, int rr, int dh, int dim) const {
        const float i1 = l[0] != 0.0f ? p.out_scale / l[0] : 0.0f, i2 = l[1] != 0.0f ? p.lambda * p.out_scale / l[1] : 0.0f;
#pragma unroll
        for (int d = 0; d < 4; d += 2) ca_write2(p, it, rr, dh, dim + d, o[0][d] * i1 - o[1][d] * i2, o[0][d + 1] * i1 - o[1][d + 1] * i2);
    }
};
// Joins n parts of an item, in order: at(j) is the j-th.  `to`: where the result stays a part, null if it is the output.  Threads deal (row, four dims).
template <int DH, int ROWS, class F>
__device__ __forceinline__ void ca_join(const CaParams &p, const CaItem &it, int n, F at, float *to, int thread, int threads) {
    constexpr int PART = 4 + 2 * DH, FOURS = DH / 4;
    const int all = ROWS * p.tiles, end = min(all, it.m * p.group - it.tile * all);
    constexpr int AT_ONCE = ROWS == 1 ? 1 : 4;  // places of a thread whose loads are in flight together
    for (int e0 = thread; e0 < end * FOURS; e0 += AT_ONCE * threads) {
        CaSum sum[AT_ONCE];
#pragma unroll 2
        for (int j = 0; j < n; ++j) {
            const float *part = at(j);
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int e = min(e0 + u * threads, end * FOURS - 1);
                sum[u].add_part(part + e / FOURS * PART, DH, e % FOURS * 4);
            }
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int e = e0 + u * threads, r = e / FOURS, dim = e % FOURS * 4;
            if (e >= end * FOURS) break;
            if (to) sum[u].store_part(to + r * PART, DH, dim, dim == 0);
            else sum[u].write(p, it, it.tile * all + r, DH, dim);
        }
    }
}

}  // namespace hgf
#include "hgf_cached_attention_tc.cuh"
namespace hgf {

template <int DH, int ROWS>
__global__ void __launch_bounds__(CaCfg<DH, ROWS>::THREADS, 1) cached_attention_kernel(CaParams p) {
    using C = CaCfg<DH, ROWS>;
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3, H = p.c.H;
    const int team_warps = ROWS == 1 ? 1 : 2 * p.tiles, team = ROWS == 1 ? warp : warp / team_warps;
    const int member = ROWS == 1 ? 0 : warp - team * team_warps, my_tile = member >> 1, stream = member & 1;
    const bool leads = member == 0;
    const int stages = ROWS == 1 ? 2 : p.stages;
    uint8_t *ring = smem + team * stages * C::STAGE;
    float *scores = reinterpret_cast<float *>(smem + C::STAGES * C::STAGE + warp * C::SCORES);
    long long *prefix = reinterpret_cast<long long *>(smem + C::STAGES * C::STAGE + C::WARPS * C::SCORES);
    __shared__ long long wide[C::WARPS];
    __shared__ __align__(8) uint64_t bars[C::STAGES];
    __shared__ int page_ok[C::STAGES];       // a stage's page number was one
    __shared__ volatile int gave_up;         // a wait ran out: the others end, too
    __shared__ int unseen;                   // there are rows that see no token
    __shared__ uint32_t odd_of[ROWS == 1 ? C::WARPS : C::WARPS / 2][2][DH];  // of a team's 64 open tokens, for each dim, those with a value that is not finite
    __shared__ volatile int odd_at[kCaMaxTeams];  // the unit of a team's share in which there last were some
    uint32_t (*odd)[DH] = odd_of[team];
    if (tid < kCaMaxTeams) odd_at[tid] = -1;
    __shared__ CaItem first_item_of_cta, last_item_of[kCaMaxTeams];
    const uint32_t ring_a = dsmem_u32(ring), bars_a = dsmem_u32(bars) + team * stages * 8;
    if (tid < C::STAGES) dmbar_init(dsmem_u32(&bars[tid]), 1);
    if (tid == 0) gave_up = unseen = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    __syncthreads();
    pdl_wait();
    pdl_launch_dependents();
    const int tile_rows = ROWS * (ROWS == 1 ? 1 : p.tiles);

    // ---- plan: the running sum of units over the sequences, by every CTA for itself
    // (up to 32 of them: by every warp for itself, without a barrier)
    long long total = 0;
    if (tid == 0) p.items[2 * blockIdx.x] = make_int4(0, 0, 0, 0);
    auto units_of = [&](int i) {
        const CaSeq s = ca_sequence(p, tile_rows, i);
        if (blockIdx.x == 0 && s.slot == -2) atomicOr(p.status, kStatusCache);
        if (s.m > s.length) unseen = 1;
        return (long long)(s.tiles - s.tile0) * H * s.units;
    };
    auto warp_sum = [&](long long sum) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        return sum;
    };
    if (p.n_seqs <= 32) {
        const long long mine = lane < p.n_seqs ? units_of(lane) : 0, sum = warp_sum(mine);
        total = __shfl_sync(0xffffffffu, sum, 31);
        if (lane < p.n_seqs) prefix[lane] = sum - mine;  // (every warp writes the same values)
        if (lane == 0) prefix[p.n_seqs] = total;
    } else {
        for (int i0 = 0; i0 < p.n_seqs; i0 += blockDim.x) {
            const int i = i0 + tid;
            const long long mine = i < p.n_seqs ? units_of(i) : 0, sum = warp_sum(mine);
            if (lane == 31) wide[warp] = sum;
            __syncthreads();
            long long before = total, all = 0;
            const int warps = blockDim.x >> 5;
            for (int w = 0; w < warps; ++w) {
                if (w < warp) before += wide[w];
                all += wide[w];
            }
            if (i < p.n_seqs) prefix[i] = before + sum - mine;
            total += all;
            __syncthreads();
        }
        if (tid == 0) prefix[p.n_seqs] = total;
        __syncthreads();
    }
    __syncwarp();

    // rows that see no token: the first of more rows than the sequence has tokens.  (A warp that has not come across one does its part all the same once
    // another has: the flag is read behind a barrier.)
    __syncthreads();
    if (unseen) {
        const int width = H * p.group * DH;
        for (int i = blockIdx.x; i < p.n_seqs; i += gridDim.x) {
            const CaSeq s = ca_sequence(p, tile_rows, i);
            const size_t at = (size_t)s.row0 * width, n = (size_t)max(s.m - s.length, 0) * width;  // (16 bytes at a time: width is a multiple of 64)
            if (p.bf16) for (size_t e = 8 * tid; e < n; e += 8 * blockDim.x) *reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(p.out) + at + e) = make_uint4(0, 0, 0, 0);
            else for (size_t e = 4 * tid; e < n; e += 4 * blockDim.x) *reinterpret_cast<uint4 *>(reinterpret_cast<float *>(p.out) + at + e) = make_uint4(0, 0, 0, 0);
        }
    }

    // ---- shares.  As many CTAs as have a unit for each team, as many teams as have a unit: none is empty between two of an item, and a short item
    // stays within a CTA.
    const int teams_here = ROWS == 1 ? C::WARPS : p.teams;
    const int ctas = total < (long long)gridDim.x * teams_here ? ((int)total + teams_here - 1) / teams_here : (int)gridDim.x;
    if ((int)blockIdx.x >= ctas) return;
    const long long c0 = ca_share(total, blockIdx.x, ctas), c1 = ca_share(total, blockIdx.x + 1, ctas);
    const int teams = (int)min((long long)teams_here, c1 - c0);
    const bool works = team < teams;
    const long long u0 = works ? c0 + ca_share(c1 - c0, team, teams) : c1, u1 = works ? c0 + ca_share(c1 - c0, team + 1, teams) : c1;
    const int part_floats = (ROWS == 1 ? 1 : p.tiles) * (ROWS * C::PART);
    float *parts = ROWS == 1 ? reinterpret_cast<float *>(smem + C::STAGES * C::STAGE + C::WARPS * C::SCORES + C::PREFIX) : p.parts + (size_t)blockIdx.x * teams_here * 2 * part_floats;
    float *my_parts = parts + team * 2 * part_floats;
    float *given = ROWS == 8 ? reinterpret_cast<float *>(smem + C::STAGES * C::STAGE + (warp & ~1) * C::SCORES)
                             : reinterpret_cast<float *>(smem + C::STAGES * C::STAGE + C::WARPS * C::SCORES + C::PREFIX) + (ROWS == 1 ? 0 : (warp >> 1) * C::GIVEN);

    auto place = [&](long long u, CaCursor &k) {
        int lo = 0, hi = p.n_seqs - 1;
        while (lo < hi) {  // the last sequence that begins at or before u (of empty ones at the same place the last, which is not empty)
            const int mid = (lo + hi + 1) >> 1;
            if (prefix[mid] <= u) lo = mid; else hi = mid - 1;
        }
        k.seq = lo;
        k.s = ca_sequence(p, tile_rows, lo);
        const long long in = u - prefix[lo];
        const long long item = in <= 0xffffffffll ? (long long)((uint32_t)in / (uint32_t)k.s.units) : in / k.s.units;
        k.unit = (int)(in - item * k.s.units);
        k.tile = item <= 0xffffffffll ? (int)((uint32_t)item / (uint32_t)H) : (int)(item / H);
        k.head = (int)(item - (long long)k.tile * H);
        k.tile += k.s.tile0;
    };
    auto advance = [&](CaCursor &k) {  // to the next unit; true: of another item
        if (++k.unit < k.s.units) return false;
        k.unit = 0;
        if (++k.head < H) return true;
        k.head = 0;
        if (++k.tile < k.s.tiles) return true;
        do ++k.seq; while (k.seq < p.n_seqs - 1 && prefix[k.seq + 1] == prefix[k.seq]);
        if (k.seq < p.n_seqs) k.s = ca_sequence(p, tile_rows, k.seq);
        k.tile = k.s.tile0;
        return true;
    };
    // The last row of an item sees the tokens before this.
    auto last_sees = [&](const CaSeq &s, int tile) {
        const int at = (tile + 1) * tile_rows - 1;
        return s.length - s.m + 1 + min(s.m - 1, p.group == 1 ? at : at / p.group);
    };
    auto unit_token = [&](const CaCursor &k) { return k.unit < k.s.pages ? k.unit << 6 : (k.s.pages << 6) + ((k.unit - k.s.pages) << 5); };
    auto team_sync = [&] {
        if (ROWS == 1) __syncwarp();
        else bar_sync(1 + team, team_warps * 32);
    };

    // ---- the ring: the leading warp fetches, page numbers 32 at a time, one bulk copy a unit
    int pages32 = 0, pages_at = -32, pages_seq = -1;
    auto fetch = [&](const CaCursor &k, int sees, int stage) {
        const uint32_t bar = bars_a + stage * 8, dst = ring_a + stage * C::STAGE;
        if (unit_token(k) >= sees) return;  // (nobody waits for it either)
        if (k.unit < k.s.pages) {
            if (pages_seq != k.seq || (k.unit & ~31) != pages_at) {
                pages_seq = k.seq;
                pages_at = k.unit & ~31;
                pages32 = pages_at + lane < k.s.pages ? p.c.table[(size_t)k.s.slot * p.c.max_pages + pages_at + lane] : 0;
            }
            const int page = __shfl_sync(0xffffffffu, pages32, k.unit & 31);
            const bool ok = page >= 0 && page < p.c.n_pages;
            if (lane == 0) {
                page_ok[team * stages + stage] = ok;
                if (ok) {
                    const size_t at = (size_t)page * H + k.head;
                    announce(bar, C::UNIT + 16);
                    bulk_load_announced(dst, p.c.codes + at * C::UNIT, C::UNIT, bar);
                    bulk_load_announced(dst + C::UNIT, p.c.scales + at, 16, bar);
                } else {
                    atomicOr(p.status, kStatusCache);
                    announce(bar, 0);
                }
            }
        } else if (lane == 0) {
            const int half = k.unit - k.s.pages, rows = min(32, (k.s.length & 63) - 32 * half);
            const __nv_bfloat16 *src = p.c.open + (((size_t)k.s.slot * H + k.head) * 3 * kCacheBlock + 32 * half) * DH;
            page_ok[team * stages + stage] = 1;
            announce(bar, 3 * rows * DH * 2);
#pragma unroll
            for (int n = 0; n < 3; ++n) bulk_load_announced(dst + n * 32 * DH * 2, src + (size_t)n * kCacheBlock * DH, rows * DH * 2, bar);
        }
    };
    uint32_t phases = 0;
    auto arrived = [&](int stage, bool last) {  // waits, bounded, for the stage's copies
        const uint32_t bar = bars_a + stage * 8, parity = phases >> stage & 1u;
        bool got = dmbar_try_wait(bar, parity);
        if (__all_sync(0xffffffffu, got)) return true;
        const unsigned long long since = dec_timer_ns();
        for (uint32_t polls = 1; !got && !(got = dmbar_try_wait(bar, parity)); ++polls)
            if ((polls & 255u) == 0 && ((!last && gave_up) || dec_timer_ns() - since > kDecWaitLimitNs)) break;
        if (!got) {
            gave_up = 1;
            atomicExch(p.status, 0xb00u);
        }
        return (bool)__all_sync(0xffffffffu, got);
    };

    CaCursor ahead, k;
    if (works) place(u0, k);
    if (works && team == 0 && lane == 0 && leads) first_item_of_cta = {u0 - k.unit, u0 - k.unit + k.s.units, k.s.row0, k.s.m, k.head, k.tile};

    // ---- state of the item
    // ROWS = 1: m, l of the lane's stream (lanes 0-15 stream 1, 16-31 stream 2); acc[mt][e]: dims 16 mt + g + 8 e, in lanes t of stream t / 2.
    // ROWS = 8: m, l of row g, of the warp's stream; acc[mt][e]: dim 16 mt + g + 8 (e / 2), row 2 t + e % 2.
    // ROWS = 16: m, l of rows g and g + 8, of the warp's stream; acc[nt][e]: dim 8 nt + 2 t + e % 2, row g + 8 (e / 2).
    constexpr int NR = ROWS == 16 ? 2 : 1, NA = ROWS == 16 ? DH / 8 : C::MT, NE = ROWS == 1 ? 2 : 4, ND = ROWS == 1 ? 1 : 3;
    float m[NR], l[NR], acc[NA][NE];
    uint32_t qd[ROWS == 1 ? 2 : ND][C::KT][ROWS == 16 ? 4 : 2];  // digits of q: ROWS = 1 for K1 and for K2, as right operand; else each digit, as right or left operand
    int sees_e[2] = {0, 0};                        // (ROWS = 8) tokens that rows 2 t and 2 t + 1 see
    float qs[NR];                                  // what a digit sum is worth, with 1 / sqrt(d) and log2 e
    int sees[NR] = {}, sees_tile = 0, sees_all = 0, sees_item = 0, sees_first = 0;  // tokens that the lane's rows, any row, every row of the tile, any of the item, its first row sees
    const int my_stream = ROWS == 1 ? lane >> 4 : stream, limb = g & 3;
    const uint32_t limb_sel = 0x0040u + (uint32_t)((2 - limb) & 3) * 0x0011u;  // byte 2 - limb of two words
    const uint32_t limb_xor = limb == 0 ? 0x80808080u : 0u, limb_keep = limb == 3 ? 0u : 0xffffffffu;
    const int heads = H * p.group;

    // Of the tile's row r: its token and its head of the group.  (One division an item: what is left is below 2^17, where a product with the rounded 1 / group
    // is off by far less than the half that it stands from the next integer.)
    struct Tile {
        int token, left;  // of its first row
    };
    auto tile_of = [&](const CaCursor &k) {
        const int at = k.tile * tile_rows + my_tile * ROWS, token = p.group == 1 ? at : at / p.group;
        return Tile{token, at - token * p.group};
    };
    auto token_of = [&](const Tile &b, int r) { return p.group == 1 ? b.token + r : b.token + (int)(((float)(b.left + r) + 0.5f) * p.per_group); };
    auto q_row = [&](const CaCursor &k, const Tile &b, int n, int r) {  // stream n of the tile's row r
        const int token = token_of(b, r);
        return p.q + ((size_t)(k.s.row0 + token) * 2 + n) * heads * DH + (size_t)(k.head * p.group + b.left + r - (token - b.token) * p.group) * DH;
    };
    Tile tile = {0, 0};  // the item's
    uint2 qw[NR][C::KT][2];                        // q's values in the places of its digits: of the lane's rows (ROWS = 1: the one row) and stream
    auto load_q = [&](const CaCursor &k, const Tile &b) {
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            const int row = ROWS == 1 ? 0 : g + 8 * r;
            const bool there = token_of(b, row) < k.s.m;
            const __nv_bfloat16 *src = q_row(k, b, my_stream, there ? row : 0) + 4 * t;
#pragma unroll
            for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
                for (int h = 0; h < 2; ++h) qw[r][kt][h] = there ? *reinterpret_cast<const uint2 *>(src + kt * 32 + h * 16) : make_uint2(0, 0);
        }
    };
    if (ROWS == 1 && works) load_q(k, tile_of(k));
    ahead = k;
    long long ahead_u = u0;
    int ahead_sees = works ? last_sees(k.s, k.tile) : 0;  // tokens that the last row of the item sees
    auto fetch_next = [&](int stage) {
        fetch(ahead, ahead_sees, stage);
        if (++ahead_u < u1 && advance(ahead)) ahead_sees = last_sees(ahead.s, ahead.tile);
    };
    if (leads)
        for (int s = 0; s < stages && ahead_u < u1; ++s) fetch_next(s);
    auto begin_item = [&] {
#pragma unroll
        for (int a = 0; a < NA; ++a)
#pragma unroll
            for (int e = 0; e < NE; ++e) acc[a][e] = 0.0f;
        tile = tile_of(k);
        if (ROWS > 1) load_q(k, tile);
        // row r sees the tokens before first + its token, if it is there
        const int first = k.s.length - k.s.m + 1;
        auto sees_of = [&](int r) {
            const int token = token_of(tile, r);
            return token < k.s.m ? first + token : 0;
        };
        sees_item = last_sees(k.s, k.tile);
        sees_first = k.s.length - k.s.m + 1 + (p.group == 1 ? k.tile * tile_rows : k.tile * tile_rows / p.group);
        if (ROWS == 1) {
            sees[0] = sees_tile = sees_all = sees_of(0);
        } else if (ROWS == 8) {
            sees[0] = sees_of(g);
            sees_e[0] = sees_of(2 * t);
            sees_e[1] = sees_of(2 * t + 1);
            sees_tile = sees_item;
            sees_all = min(sees_of(0), sees_of(7));
        } else {
            sees[0] = sees_of(g);
            sees[NR - 1] = sees_of(g + 8);
            sees_tile = tile.token < k.s.m ? first + min(k.s.m - 1, token_of(tile, 15)) : 0;
            sees_all = min(sees_of(0), sees_of(15));
        }
        // q's digits: q = f * 2^(E - 21) with E the exponent of the row's largest magnitude, so |f| < 2^22; f + 0x808080 has in each byte the
        // balanced digit plus 128.  (f is rounded by adding 1.5 * 2^23.)
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.0f;
            uint32_t top = 0;
#pragma unroll
            for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
                for (int h = 0; h < 2; ++h) top = __vmaxu2(top, __vmaxu2(qw[r][kt][h].x & 0x7fff7fffu, qw[r][kt][h].y & 0x7fff7fffu));
            top = max(top >> 16, top & 0xffffu);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int E = max((int)(top >> 7) - 127, -100);  // (below 2^-100 the scores are zero for any purpose, above that 2^(21 - E) is a float)
            const float f = __uint_as_float((uint32_t)(127 + 21 - E) << 23);
            const float back = top >= 0x7f80u ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)(127 - 21 + E) << 23);
            qs[r] = back * p.scale_log2;
#pragma unroll
            for (int kt = 0; kt < C::KT; ++kt)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint2 w = qw[r][kt][h];
                    const float v[4] = {bf16lo_to_float(w.x), bf16hi_to_float(w.x), bf16lo_to_float(w.y), bf16hi_to_float(w.y)};
                    uint32_t d[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[e] = __float_as_uint(fmaf(v[e], f, kCaMagicF)) + (0x808080u - 0x400000u);
                    if (ROWS == 1) {
                        const uint32_t x = (__byte_perm(__byte_perm(d[0], d[1], limb_sel), __byte_perm(d[2], d[3], limb_sel), 0x5410) ^ 0x80808080u) & limb_keep;
                        qd[0][kt][h] = my_stream ? 0u : x;
                        qd[1][kt][h] = my_stream ? x : 0u;
                    } else {
#pragma unroll
                        for (int j = 0; j < ND; ++j) {
                            const uint32_t sel = 0x0040u + (uint32_t)(2 - j) * 0x0011u;
                            qd[j][kt][ROWS == 16 ? 2 * h + r : h] = __byte_perm(__byte_perm(d[0], d[1], sel), __byte_perm(d[2], d[3], sel), 0x5410) ^ 0x80808080u;
                        }
                    }
                }
        }
    };

    // Softmax step of row r on `x`, scores before their factor f (16 or 8 tokens of this lane, the row's others in the lanes with the same g; the first
    // `count` of the unit's tokens count, `token(j)` is the j-th of the lane's): the probabilities relative to the unit's largest in place of the scores,
    // and what the sums so far (alpha) and the unit's (worth) are to be multiplied with.
    auto softmax_step = [&](auto &x, int r, float f, bool partly, int count, auto token, float &alpha, float &worth) {
        constexpr int N = sizeof(x) / sizeof(float);
        if (partly) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (token(j) >= count) x[j] = -INFINITY;
        }
        float tops[4] = {x[0], x[1], x[2], x[3]}, sums[4] = {};  // (four chains: a dependent operation waits four clocks)
#pragma unroll
        for (int j = 4; j < N; ++j) tops[j & 3] = fmaxf(tops[j & 3], x[j]);
        float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        f = count > 0 ? f + 1.17549435e-38f : 1.0f;  // (a page of zeros has f = 0, one that the row sees nothing of may have NaN, and what is masked has to stay at -inf)
        const float here = top * f, now = fmaxf(m[r], here), base = now == -INFINITY ? 0.0f : now;
        const float minus = top == -INFINITY ? 0.0f : -top;
        const uint64_t minus2 = pack_f32x2(minus, minus), f2 = pack_f32x2(f, f);
        alpha = exp2_approx(m[r] - base);
        worth = exp2_approx(here - base);
        // (the difference first: the largest gives exactly 1, however large the scores)
#pragma unroll
        for (int j = 0; j < N; j += 2) {
            unpack_f32x2(mul_f32x2(add_f32x2(pack_f32x2(x[j], x[j + 1]), minus2), f2), x[j], x[j + 1]);
            x[j] = exp2_approx(x[j]);
            x[j + 1] = exp2_approx(x[j + 1]);
            sums[j & 3] += x[j];
            sums[(j + 1) & 3] += x[j + 1];
        }
        m[r] = now;
        l[r] = fmaf(l[r], alpha, ((sums[0] + sums[1]) + (sums[2] + sums[3])) * worth);
    };

    int magic[4] = {(int)kCaMagic, (int)kCaMagic, (int)kCaMagic, (int)kCaMagic};
    const bool begins_inside = works && k.unit != 0;  // the share's first item began in another share
    bool fresh = true, first_item = true, has_next = false;
    CaCursor next;
    // A warp whose wait ran out computes and fetches no more, but takes its steps to the end: the others of its team meet it at their barrier.
    bool dead = false;
    int odd_halves = 0;  // the item's open units that had values which are not finite taken out
    int stage = 0;
    for (long long u = u0; u < u1; ++u) {
        if (fresh) begin_item();
        // (the next item's q is on its way while this one's last units are worked on)
        const bool item_ends = k.unit == k.s.units - 1;
        if (ROWS == 1 && !has_next && k.unit >= k.s.units - 2 && u + (k.s.units - k.unit) < u1) {
            next = k;
            next.unit = k.s.units - 1;
            advance(next);
            load_q(next, tile_of(next));
            has_next = true;
        }
        const uint8_t *unit = ring + stage * C::STAGE;
        const int token0 = unit_token(k);
        if (token0 < sees_item) {
            if (!dead) {
                if (arrived(stage, false)) {
                    phases ^= 1u << stage;
                } else {
                    dead = true;
                    if (leads)  // (no copy outlives the CTA)
                        for (int s = 0; u + s < ahead_u; ++s) arrived((stage + s) % stages, true);
                }
            }
            const bool ok = !dead && page_ok[team * stages + stage];
            const bool open_unit = k.unit >= k.s.pages;
            if (open_unit) {
                // what lies behind the last row is no value: V's rows there become zero (K's only give scores that are not looked at)
                const int rows = min(32, (k.s.length & 63) - 32 * (k.unit - k.s.pages));
                uint8_t *mine = ring + stage * C::STAGE;
                if (leads)
                    for (int e = lane; e < (32 - rows) * (DH / 8); e += 32) *reinterpret_cast<uint4 *>(mine + 2 * 32 * DH * 2 + rows * DH * 2 + e * 16) = make_uint4(0, 0, 0, 0);
                // Where a row sees some of these tokens and not all, zero times a value that is not finite would reach it: such values become zero here, and
                // odd[.][dim] says of which tokens there were some.  (Looked for in a wide pass first: there are none.)
                const bool some = sees_first < token0 + rows;
                __nv_bfloat16 *values = reinterpret_cast<__nv_bfloat16 *>(mine + 2 * 32 * DH * 2);
                if (some) {
                    uint32_t top = 0;
                    for (int e = member * 32 + lane; e < rows * (DH / 8); e += team_warps * 32) {
                        const uint4 w = reinterpret_cast<const uint4 *>(values)[e];
                        top = __vmaxu2(top, __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu)));
                    }
                    if (max(top >> 16, top & 0xffffu) >= 0x7f80u) odd_at[team] = (int)(u - u0);
                }
                team_sync();
                if (some && odd_at[team] == (int)(u - u0)) {
                    const int half = k.unit - k.s.pages;
                    odd_halves |= 1 << half;
                    for (int dim = member * 32 + lane; dim < DH; dim += team_warps * 32) {
                        uint32_t which = 0;
                        for (int r = 0; r < rows; ++r) {
                            __nv_bfloat16 &x = values[r * DH + cache_open_eight(r, dim >> 3) * 8 + (dim & 7)];
                            if ((__bfloat16_as_ushort(x) & 0x7f80) != 0x7f80) continue;
                            which |= 1u << r;
                            x = __ushort_as_bfloat16(0);
                        }
                        odd[half][dim] = which;
                    }
                    team_sync();
                }
            }
            if (ok && !open_unit && token0 < sees_tile) {
                const float4 sc = *reinterpret_cast<const float4 *>(unit + C::UNIT);
                auto token = [&](int j) { return (j >> 2) * 16 + 4 * t + (j & 3); };
                const bool partly = sees_all - token0 < kCacheBlock;
                float x[NR][16], alpha[NR], worth[NR];
                if constexpr (ROWS == 1) {
                    const float wa = t & 1 ? 1.0f : 65536.0f, wb = t & 1 ? 0.0f : 256.0f;
#pragma unroll
                    for (int mt = 0; mt < 4; ++mt) {
                        int d[4];
#pragma unroll
                        for (int n = 0; n < 2; ++n)
#pragma unroll
                            for (int kt = 0; kt < C::KT; ++kt) {
                                const uint4 a = *reinterpret_cast<const uint4 *>(unit + n * kCacheBlock * DH + ((mt * C::KT + kt) * 32 + lane) * 16);
                                mma_s8s8(d, a, qd[n][kt][0], qd[n][kt][1], n + kt ? d : magic);
                            }
                        float lo = fmaf(ca_float(d[0]), wa, ca_float(d[1]) * wb), hi = fmaf(ca_float(d[2]), wa, ca_float(d[3]) * wb);
                        lo += __shfl_xor_sync(0xffffffffu, lo, 1);
                        hi += __shfl_xor_sync(0xffffffffu, hi, 1);
                        scores[(t >> 1) * kCacheBlock + mt * 16 + g + (t & 1) * 8] = t & 1 ? hi : lo;
                    }
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float4 v = *reinterpret_cast<const float4 *>(scores + my_stream * kCacheBlock + j * 16 + 4 * t);
                        x[0][4 * j] = v.x;
                        x[0][4 * j + 1] = v.y;
                        x[0][4 * j + 2] = v.z;
                        x[0][4 * j + 3] = v.w;
                    }
                    softmax_step(x[0], 0, qs[0] * (my_stream ? sc.y : sc.x), partly, sees[0] - token0, token, alpha[0], worth[0]);
                    uint32_t b[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(1.0f + x[0][4 * j + e]);
                        b[j] = (__byte_perm(__byte_perm(w[0], w[1], limb_sel), __byte_perm(w[2], w[3], limb_sel), 0x5410) ^ limb_xor) & limb_keep;
                    }
                    const float scale = __shfl_sync(0xffffffffu, alpha[0], (t >> 1) * 16), sv = sc.z * __shfl_sync(0xffffffffu, worth[0], (t >> 1) * 16);
                    // digits of 2^23 p: weights 2^-7, 2^-15, 2^-23
                    const float va = sv * (t & 1 ? 1.1920928955078125e-7f : 0.0078125f), vb = t & 1 ? 0.0f : sv * 3.0517578125e-5f;
#pragma unroll
                    for (int mt = 0; mt < C::MT; ++mt) {
                        int d[4];
#pragma unroll
                        for (int kt = 0; kt < 2; ++kt) {
                            const uint4 a = *reinterpret_cast<const uint4 *>(unit + 2 * kCacheBlock * DH + ((mt * 2 + kt) * 32 + lane) * 16);
                            mma_s8u8(d, a, b[2 * kt], b[2 * kt + 1], kt ? d : magic);
                        }
                        acc[mt][0] = fmaf(ca_float(d[0]), va, fmaf(ca_float(d[1]), vb, acc[mt][0] * scale));
                        acc[mt][1] = fmaf(ca_float(d[2]), va, fmaf(ca_float(d[3]), vb, acc[mt][1] * scale));
                    }
                } else if constexpr (ROWS == 8) {
                    const uint64_t base256 = pack_f32x2(256.0f, 256.0f);
                    const uint8_t *codes = unit + stream * kCacheBlock * DH;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
#pragma unroll
                        for (int mh = 0; mh < 2; ++mh) {
                            const int mt = 2 * half + mh;
                            int d[3][4];
#pragma unroll
                            for (int kt = 0; kt < C::KT; ++kt) {
                                const uint4 a = *reinterpret_cast<const uint4 *>(codes + ((mt * C::KT + kt) * 32 + lane) * 16);
#pragma unroll
                                for (int z = 0; z < 3; ++z) mma_s8s8(d[z], a, qd[z][kt][0], qd[z][kt][1], kt ? d[z] : magic);
                            }
#pragma unroll
                            for (int e = 0; e < 4; e += 2) {
                                float v0, v1;
                                unpack_f32x2(fma_f32x2(fma_f32x2(ca_float2(d[0][e], d[0][e + 1]), base256, ca_float2(d[1][e], d[1][e + 1])), base256, ca_float2(d[2][e], d[2][e + 1])), v0, v1);
                                scores[2 * t * 36 + mh * 16 + g + 4 * e] = v0;
                                scores[2 * t * 36 + 36 + mh * 16 + g + 4 * e] = v1;
                            }
                        }
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const float4 v = *reinterpret_cast<const float4 *>(scores + g * 36 + j * 16 + 4 * t);
                            x[0][8 * half + 4 * j] = v.x;
                            x[0][8 * half + 4 * j + 1] = v.y;
                            x[0][8 * half + 4 * j + 2] = v.z;
                            x[0][8 * half + 4 * j + 3] = v.w;
                        }
                        __syncwarp();
                    }
                    softmax_step(x[0], 0, qs[0] * (stream ? sc.y : sc.x), partly, sees[0] - token0, token, alpha[0], worth[0]);
                    uint32_t pd[3][4];  // digits of the probabilities, as right operand
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(1.0f + x[0][4 * j + e]);
                        pd[0][j] = __byte_perm(__byte_perm(w[0], w[1], 0x0062), __byte_perm(w[2], w[3], 0x0062), 0x5410) ^ 0x80808080u;
                        const uint32_t w01 = __byte_perm(w[0], w[1], 0x5140), w23 = __byte_perm(w[2], w[3], 0x5140);
                        pd[1][j] = __byte_perm(w01, w23, 0x7632);
                        pd[2][j] = __byte_perm(w01, w23, 0x5410);
                    }
                    // (a row that sees none of the page takes nothing of it, not even a scale that is NaN)
                    constexpr float kUnit = 1.1920928955078125e-7f;
                    float scale[2], sv[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        scale[e] = __shfl_sync(0xffffffffu, alpha[0], (2 * t + e) * 4);
                        sv[e] = __shfl_sync(0xffffffffu, worth[0], (2 * t + e) * 4);
                        sv[e] = sees_e[e] > token0 ? sv[e] * sc.z * kUnit : 0.0f;
                    }
                    const uint64_t scale2 = pack_f32x2(scale[0], scale[1]), sv2 = pack_f32x2(sv[0], sv[1]);
#pragma unroll
                    for (int mt = 0; mt < C::MT; ++mt) {
                        int d[3][4];
#pragma unroll
                        for (int kt = 0; kt < 2; ++kt) {
                            const uint4 a = *reinterpret_cast<const uint4 *>(unit + 2 * kCacheBlock * DH + ((mt * 2 + kt) * 32 + lane) * 16);
#pragma unroll
                            for (int z = 0; z < 3; ++z) mma_s8u8(d[z], a, pd[z][2 * kt], pd[z][2 * kt + 1], kt ? d[z] : magic);
                        }
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            uint64_t y = fma_f32x2(ca_float2(d[0][e], d[0][e + 1]), base256, ca_float2(d[1][e], d[1][e + 1]));
                            y = fma_f32x2(y, base256, ca_float2(d[2][e], d[2][e + 1]));
                            unpack_f32x2(fma_f32x2(y, sv2, mul_f32x2(pack_f32x2(acc[mt][e % NE], acc[mt][(e + 1) % NE]), scale2)), acc[mt][e % NE], acc[mt][(e + 1) % NE]);
                        }
                    }
                } else {
                    const uint64_t base256 = pack_f32x2(256.0f, 256.0f);
                    // Column n of a product is token 4 (n / 2) + n % 2 of sixteen, or the one two further: a lane's two columns are then its first or
                    // last two of four neighbouring tokens.  In the tile such a token's row is 8 a + g' with a = n / 4.
                    const uint8_t *codes = unit + stream * kCacheBlock * DH + (((g & 1) + 4 * (g >> 1 & 1)) * 4 + t) * 16 + (g >> 2) * 4;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
#pragma unroll
                        for (int two = 0; two < 2; ++two) {
                            int d[3][4];
#pragma unroll
                            for (int kt = 0; kt < C::KT; ++kt) {
                                const uint8_t *at = codes + (j * C::KT + kt) * 512 + two * 128;
                                const uint32_t b0 = *reinterpret_cast<const uint32_t *>(at), b1 = *reinterpret_cast<const uint32_t *>(at + 8);
#pragma unroll
                                for (int z = 0; z < 3; ++z) mma_s8s8(d[z], make_uint4(qd[z][kt][0], qd[z][kt][1], qd[z][kt][ROWS == 16 ? 2 : 0], qd[z][kt][ROWS == 16 ? 3 : 0]), b0, b1, kt ? d[z] : magic);
                            }
#pragma unroll
                            for (int r = 0; r < NR; ++r)
                                unpack_f32x2(fma_f32x2(fma_f32x2(ca_float2(d[0][2 * r], d[0][2 * r + 1]), base256, ca_float2(d[1][2 * r], d[1][2 * r + 1])), base256,
                                                       ca_float2(d[2][2 * r], d[2][2 * r + 1])),
                                             x[r][4 * j + 2 * two], x[r][4 * j + 2 * two + 1]);
                        }
                    const float sk = stream ? sc.y : sc.x;
                    uint32_t pd[3][2][4];  // digits of the probabilities, as left operand of the two products over 32 tokens
                    uint64_t scale2[NR], sv2[NR];
                    constexpr float kUnit = 1.1920928955078125e-7f;
#pragma unroll
                    for (int r = 0; r < NR; ++r) {
                        softmax_step(x[r], r, qs[r] * sk, partly, sees[r] - token0, token, alpha[r], worth[r]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            uint32_t w[4];
                            const int kt = j >> 1, at = 2 * (j & 1) + r;
#pragma unroll
                            for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(1.0f + x[r][4 * j + e]);
                            pd[0][kt][at] = __byte_perm(__byte_perm(w[0], w[1], 0x0062), __byte_perm(w[2], w[3], 0x0062), 0x5410) ^ 0x80808080u;
                            const uint32_t w01 = __byte_perm(w[0], w[1], 0x5140), w23 = __byte_perm(w[2], w[3], 0x5140);
                            pd[1][kt][at] = __byte_perm(w01, w23, 0x7632);
                            pd[2][kt][at] = __byte_perm(w01, w23, 0x5410);
                        }
                        // (a row that sees none of the page takes nothing of it, not even a scale that is NaN)
                        const float sv = sees[r] > token0 ? worth[r] * sc.z * kUnit : 0.0f;
                        scale2[r] = pack_f32x2(alpha[r], alpha[r]);
                        sv2[r] = pack_f32x2(sv, sv);
                    }
#pragma unroll
                    for (int mt = 0; mt < C::MT; ++mt) {
                        uint4 v[2];
#pragma unroll
                        for (int kt = 0; kt < 2; ++kt) v[kt] = *reinterpret_cast<const uint4 *>(unit + 2 * kCacheBlock * DH + ((mt * 2 + kt) * 32 + lane) * 16);
#pragma unroll
                        for (int a = 0; a < 2; ++a) {
                            int d[3][4];
                            float (&o)[NE] = acc[ROWS == 16 ? 2 * mt + a : 0];
#pragma unroll
                            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                                for (int z = 0; z < 3; ++z) mma_u8s8(d[z], pd[z][kt], a ? v[kt].y : v[kt].x, a ? v[kt].w : v[kt].z, kt ? d[z] : magic);
#pragma unroll
                            for (int r = 0; r < NR; ++r) {
                                uint64_t y = fma_f32x2(ca_float2(d[0][2 * r], d[0][2 * r + 1]), base256, ca_float2(d[1][2 * r], d[1][2 * r + 1]));
                                y = fma_f32x2(y, base256, ca_float2(d[2][2 * r], d[2][2 * r + 1]));
                                unpack_f32x2(fma_f32x2(y, sv2[r], mul_f32x2(pack_f32x2(o[(2 * r) % NE], o[(2 * r + 1) % NE]), scale2[r])), o[(2 * r) % NE], o[(2 * r + 1) % NE]);
                            }
                        }
                    }
                }
            } else if (ok && open_unit && token0 < sees_tile) {
                // ---- 32 open tokens
                const int rows = min(32, (k.s.length & 63) - 32 * (k.unit - k.s.pages));
                const uint32_t at = ring_a + stage * C::STAGE;
                auto token = [&](int j) { return (j >> 1) * 8 + 2 * t + (j & 1); };
                float x[NR][8], alpha[NR], worth[NR];
                uint32_t qb[NR][DH / 16][2];  // q's values as pairs
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    const int row = ROWS == 1 ? 0 : g + 8 * r;
                    const bool there = ROWS == 1 ? !limb : token_of(tile, row) < k.s.m;
                    const __nv_bfloat16 *src = q_row(k, tile, my_stream, there ? row : 0) + 2 * t;
#pragma unroll
                    for (int kt = 0; kt < DH / 16; ++kt)
#pragma unroll
                        for (int h = 0; h < 2; ++h) qb[r][kt][h] = there ? *reinterpret_cast<const uint32_t *>(src + kt * 16 + 8 * h) : 0u;
                }
                // p as a sum of three bf16, each the rounding of what the ones before leave
                auto three = [&](float a0, float a1, uint32_t (&w)[3]) {
#pragma unroll
                    for (int z = 0; z < 3; ++z) {
                        const __nv_bfloat162 v = __floats2bfloat162_rn(a0, a1);
                        w[z] = *reinterpret_cast<const uint32_t *>(&v);
                        a0 -= bf16lo_to_float(w[z]);
                        a1 -= bf16hi_to_float(w[z]);
                    }
                };
                auto v_four = [&](int i, int kt) {  // dims 16 i .. 16 i + 15 of sixteen tokens, as four 8 x 8: (dims 0-7, tokens 0-7), (8-15, 0-7), (0-7, 8-15), (8-15, 8-15)
                    const int r = kt * 16 + (lane & 7) + (lane >> 4) * 8;
                    return ldmatrix4_trans(at + 2 * 32 * DH * 2 + r * DH * 2 + cache_open_eight(r, i * 2 + (lane >> 3 & 1)) * 16);
                };
                // (a query that is not finite: its digits mean nothing, but the products of its bf16 values do; qs is NaN then)
                if constexpr (ROWS != 16) {
                    auto k_eight = [&](int n, int mt, int kt) {
                        const int r = mt * 16 + (lane & 15);
                        return ldmatrix4(at + n * 32 * DH * 2 + r * DH * 2 + cache_open_eight(r, kt * 2 + (lane >> 4)) * 16);
                    };
                    float d[2][4] = {};
#pragma unroll
                    for (int n = 0; n < (ROWS == 1 ? 2 : 1); ++n) {
                        float one[2][4] = {};
#pragma unroll
                        for (int kt = 0; kt < DH / 16; ++kt)
#pragma unroll
                            for (int mt = 0; mt < 2; ++mt) mma_bf16(one[mt], k_eight(ROWS == 1 ? n : stream, mt, kt), qb[0][kt][0], qb[0][kt][1]);
                        // (ROWS = 1: of each stream's keys, its columns)
#pragma unroll
                        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (ROWS == 8 || t >> 1 == n) d[mt][e] = one[mt][e];
                    }
#pragma unroll
                    for (int mt = 0; mt < 2; ++mt) {
                        if (ROWS == 8) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) scores[(2 * t + (e & 1)) * 36 + mt * 16 + g + (e >> 1) * 8] = d[mt][e];
                        } else if (!(t & 1)) {
                            scores[(t >> 1) * kCacheBlock + mt * 16 + g] = d[mt][0];
                            scores[(t >> 1) * kCacheBlock + mt * 16 + g + 8] = d[mt][2];
                        }
                    }
                    __syncwarp();
                    const float *row = scores + (ROWS == 8 ? g * 36 : my_stream * kCacheBlock);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 v = *reinterpret_cast<const float2 *>(row + 8 * j + 2 * t);
                        x[0][2 * j] = v.x;
                        x[0][2 * j + 1] = v.y;
                    }
                    __syncwarp();
                    softmax_step(x[0], 0, qs[0] == qs[0] ? p.scale_log2 : qs[0], true, min(rows, sees[0] - token0), token, alpha[0], worth[0]);
                    uint32_t b[3][2][2];  // (ROWS = 1: the lane's digit, in the first)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t w[3];
                        three(x[0][2 * j], x[0][2 * j + 1], w);
                        if (ROWS == 8) {
#pragma unroll
                            for (int z = 0; z < 3; ++z) b[z][j >> 1][j & 1] = w[z];
                        } else {
                            b[0][j >> 1][j & 1] = limb == 0 ? w[0] : limb == 1 ? w[1] : limb == 2 ? w[2] : 0u;
                        }
                    }
                    if constexpr (ROWS == 1) {
                        const float scale = __shfl_sync(0xffffffffu, alpha[0], (t >> 1) * 16), sv = __shfl_sync(0xffffffffu, worth[0], (t >> 1) * 16);
#pragma unroll
                        for (int mt = 0; mt < C::MT; ++mt) {
                            float o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                            for (int kt = 0; kt < 2; ++kt) mma_bf16(o, v_four(mt, kt), b[0][kt][0], b[0][kt][1]);
                            acc[mt][0] = fmaf(t & 1 ? o[0] : o[0] + o[1], sv, acc[mt][0] * scale);
                            acc[mt][1] = fmaf(t & 1 ? o[2] : o[2] + o[3], sv, acc[mt][1] * scale);
                        }
                    } else {
                        float scale[2], sv[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            scale[e] = __shfl_sync(0xffffffffu, alpha[0], (2 * t + e) * 4);
                            sv[e] = __shfl_sync(0xffffffffu, worth[0], (2 * t + e) * 4);
                        }
#pragma unroll
                        for (int mt = 0; mt < C::MT; ++mt) {
                            float o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                            for (int kt = 0; kt < 2; ++kt) {
                                const uint4 v = v_four(mt, kt);
#pragma unroll
                                for (int z = 0; z < 3; ++z) mma_bf16(o, v, b[z][kt][0], b[z][kt][1]);
                            }
                            // (a row that sees none of these tokens takes nothing of them, not even a value that is NaN)
#pragma unroll
                            for (int e = 0; e < NE; ++e)
                                if (sees_e[e & 1] > token0) acc[mt][e] = fmaf(o[e], sv[e & 1], acc[mt][e] * scale[e & 1]);
                        }
                    }
                } else {
#pragma unroll
                    for (int two = 0; two < 2; ++two) {  // sixteen tokens
                        float d[2][4] = {};
#pragma unroll
                        for (int kt = 0; kt < DH / 16; ++kt) {
                            const int r = two * 16 + (lane & 7) + (lane >> 4) * 8;  // (tokens 0-7, dims 0-7), (0-7, 8-15), (8-15, 0-7), (8-15, 8-15)
                            const uint4 kk = ldmatrix4(at + stream * 32 * DH * 2 + r * DH * 2 + cache_open_eight(r, kt * 2 + (lane >> 3 & 1)) * 16);
                            const uint4 a = make_uint4(qb[0][kt][0], qb[NR - 1][kt][0], qb[0][kt][1], qb[NR - 1][kt][1]);
                            mma_bf16(d[0], a, kk.x, kk.y);
                            mma_bf16(d[1], a, kk.z, kk.w);
                        }
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) x[ROWS == 16 ? e >> 1 : 0][4 * two + 2 * i + (e & 1)] = d[i][e];
                    }
                    uint32_t b[2][3][4];  // the probabilities' three, as left operand of the products over sixteen tokens
#pragma unroll
                    for (int r = 0; r < NR; ++r) {
                        softmax_step(x[r], r, qs[r] == qs[r] ? p.scale_log2 : qs[r], true, min(rows, sees[r] - token0), token, alpha[r], worth[r]);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            uint32_t w[3];
                            three(x[r][2 * j], x[r][2 * j + 1], w);
#pragma unroll
                            for (int z = 0; z < 3; ++z) b[j >> 1][z][2 * (j & 1) + r] = w[z];
                        }
                    }
#pragma unroll
                    for (int mt = 0; mt < C::MT; ++mt) {
                        float o[2][4] = {};
#pragma unroll
                        for (int kt = 0; kt < 2; ++kt) {
                            const uint4 v = v_four(mt, kt);
#pragma unroll
                            for (int z = 0; z < 3; ++z) {
                                const uint4 a = make_uint4(b[kt][z][0], b[kt][z][1], b[kt][z][2], b[kt][z][3]);
                                mma_bf16(o[0], a, v.x, v.z);
                                mma_bf16(o[1], a, v.y, v.w);
                            }
                        }
                        // (a row that sees none of these tokens takes nothing of them, not even a value that is NaN)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int e = 0; e < NE; ++e) {
                                float &y = acc[ROWS == 16 ? 2 * mt + i : 0][e];
                                if (sees[(e >> 1) % NR] > token0) y = fmaf(o[i][e], worth[(e >> 1) % NR], y * alpha[(e >> 1) % NR]);
                            }
                    }
                }
            }
            if (open_unit) asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");  // (the next copy into the stage comes after the zeros)
        }
        team_sync();
        if (leads && !dead && ahead_u < u1) fetch_next(stage);
        if (++stage == stages) stage = 0;

        // ---- the item's end, or the share's
        if (item_ends || u + 1 == u1) {
            const bool whole = item_ends && !(first_item && begins_inside);
            float *part = my_parts + (first_item ? 0 : part_floats) + my_tile * (ROWS * C::PART);
            const CaItem it = {u - k.unit, u - k.unit + k.s.units, k.s.row0, k.s.m, k.head, k.tile};
            if (u + 1 == u1 && leads && lane == 0) last_item_of[team] = it;
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
                l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
            }
            if constexpr (ROWS == 1) {
                const float l1 = __shfl_sync(0xffffffffu, l[0], 0), l2 = __shfl_sync(0xffffffffu, l[0], 16);
                const float m1 = __shfl_sync(0xffffffffu, m[0], 0), m2 = __shfl_sync(0xffffffffu, m[0], 16);
                float i1 = 0.0f, i2 = 0.0f;
                if (whole) {
                    i1 = l1 != 0.0f ? p.out_scale / l1 : 0.0f;
                    i2 = l2 != 0.0f ? p.lambda * p.out_scale / l2 : 0.0f;
                }
#pragma unroll
                for (int mt = 0; mt < C::MT; ++mt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float v = acc[mt][e];
                        v += __shfl_xor_sync(0xffffffffu, v, 1);
                        const float other = __shfl_xor_sync(0xffffffffu, v, 2);  // in lanes t = 0: stream 2's
                        const int dim = mt * 16 + g + 8 * e;
                        if (whole) {
                            if (t == 0) ca_write(p, it, k.tile, DH, dim, v * i1 - other * i2);
                        } else if (!(t & 1)) {
                            part[4 + (t >> 1) * DH + dim] = v;
                        }
                    }
                if (!whole && lane == 0) *reinterpret_cast<float4 *>(part) = make_float4(m1, l1, m2, l2);
            } else if constexpr (ROWS == 8) {
                if (!whole) {
                    if (t == 0) *reinterpret_cast<float2 *>(part + g * C::PART + 2 * stream) = make_float2(m[0], l[0]);
#pragma unroll
                    for (int mt = 0; mt < C::MT; ++mt)
#pragma unroll
                        for (int e = 0; e < NE; ++e) part[(2 * t + (e & 1)) * C::PART + 4 + stream * DH + mt * 16 + g + 8 * (e >> 1)] = acc[mt][e];
                } else {  // the second stream's warp gives its sums, as they enter the output, to the first's
                    const float mine = l[0] != 0.0f ? (stream ? p.lambda : 1.0f) * p.out_scale / l[0] : 0.0f;
                    float inv[2];
                    size_t row[2];
                    bool there[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        inv[e] = __shfl_sync(0xffffffffu, mine, (2 * t + e) * 4);
                        const int token = token_of(tile, 2 * t + e);
                        there[e] = token < k.s.m;
                        row[e] = ((size_t)(k.s.row0 + token) * heads + k.head * p.group + tile.left + 2 * t + e - (token - tile.token) * p.group) * DH;
                    }
#pragma unroll
                    for (int part64 = 0; part64 < DH / 64; ++part64) {
                        if (part64) team_sync();
                        if (stream)
#pragma unroll
                            for (int a = 0; a < 4; ++a)
#pragma unroll
                                for (int e = 0; e < NE; ++e) given[(2 * t + (e & 1)) * 68 + a * 16 + g + 8 * (e >> 1)] = acc[4 * part64 + a][e] * inv[e & 1];
                        team_sync();
                        if (!stream)
#pragma unroll
                            for (int a = 0; a < 4; ++a)
#pragma unroll
                                for (int e = 0; e < NE; ++e) {
                                    const int dim = a * 16 + g + 8 * (e >> 1);
                                    const float y = acc[4 * part64 + a][e] * inv[e & 1] - given[(2 * t + (e & 1)) * 68 + dim];
                                    if (!there[e & 1]) continue;
                                    const size_t o = row[e & 1] + 64 * part64 + dim;
                                    if (p.bf16) reinterpret_cast<__nv_bfloat16 *>(p.out)[o] = __float2bfloat16(y);
                                    else reinterpret_cast<float *>(p.out)[o] = y;
                                }
                    }
                    team_sync();  // (the room is that of the scores)
                }
            } else {
                float inv[NR];
#pragma unroll
                for (int r = 0; r < NR; ++r) {
                    inv[r] = l[r] != 0.0f ? (stream ? p.lambda : 1.0f) * p.out_scale / l[r] : 0.0f;
                    if (!whole) {
                        float *mine = part + (g + 8 * r) * C::PART;
                        if (t == 0) *reinterpret_cast<float2 *>(mine + 2 * stream) = make_float2(m[r], l[r]);
#pragma unroll
                        for (int a = 0; a < NA; ++a) *reinterpret_cast<float2 *>(mine + 4 + stream * DH + 8 * a + 2 * t) = make_float2(acc[a][(2 * r) % NE], acc[a][(2 * r + 1) % NE]);
                    }
                }
                if (whole) {  // the second stream's warps give theirs, as they enter the output, to the first's
#pragma unroll
                    for (int part64 = 0; part64 < DH / 64; ++part64) {
                        if (part64) team_sync();
                        if (stream)
#pragma unroll
                            for (int r = 0; r < NR; ++r)
#pragma unroll
                                for (int a = 0; a < 8; ++a) {
                                    const float *o = acc[ROWS == 16 ? 8 * part64 + a : 0];
                                    *reinterpret_cast<float2 *>(given + (g + 8 * r) * 68 + 8 * a + 2 * t) = make_float2(o[(2 * r) % NE] * inv[r], o[(2 * r + 1) % NE] * inv[r]);
                                }
                        team_sync();
                        if (!stream)
#pragma unroll
                            for (int r = 0; r < NR; ++r) {
                                const int token = token_of(tile, g + 8 * r);
                                if (token >= k.s.m) continue;
                                const size_t row = (size_t)(k.s.row0 + token) * heads + k.head * p.group + tile.left + g + 8 * r - (token - tile.token) * p.group;
#pragma unroll
                                for (int a = 0; a < 8; ++a) {
                                    const float *o = acc[ROWS == 16 ? 8 * part64 + a : 0];
                                    const float2 other = *reinterpret_cast<const float2 *>(given + (g + 8 * r) * 68 + 8 * a + 2 * t);
                                    ca_put2(p, row * DH + 64 * part64 + 8 * a + 2 * t, o[(2 * r) % NE] * inv[r] - other.x, o[(2 * r + 1) % NE] * inv[r] - other.y);
                                }
                            }
                    }
                }
            }
            if (odd_halves) {  // what was left out of the sums, in their place
                team_sync();
                const float nan = __uint_as_float(0x7fc00000u);
                for (int e = member * 32 + lane; e < tile_rows * DH; e += team_warps * 32) {
                    const int r = e / DH, dim = e % DH, token = (k.tile * tile_rows + r) / p.group, seen = k.s.length - k.s.m + 1 + token - 64 * k.s.pages;
                    bool bad = false;
                    for (int half = 0; half < 2; ++half)
                        if (odd_halves >> half & 1 && seen > 32 * half) bad |= (odd[half][dim] & 0xffffffffu >> (32 - min(seen - 32 * half, 32))) != 0;
                    if (token >= k.s.m || !bad) continue;
                    float *row = my_parts + (first_item ? 0 : part_floats) + r * C::PART + 4;
                    if (whole) ca_write(p, it, k.tile * tile_rows + r, DH, dim, nan);
                    else row[dim] = row[DH + dim] = nan;
                }
                team_sync();
                odd_halves = 0;
            }
            first_item = false;
        }
        fresh = item_ends;
        if (ROWS == 1) {
            if (item_ends && u + 1 < u1) {
                k = next;
                has_next = false;
            } else {
                ++k.unit;
            }
        } else if (u + 1 < u1) {
            advance(k);
        }
    }

    // ---- items that teams of this CTA share
    __syncthreads();
    if (!works) return;
    auto team_of = [&](long long unit) { return ca_share_of(c1 - c0, unit - c0, teams); };
    auto join_here = [&](const CaItem &it, int from, bool slot1, float *to) {
        const float *base = parts + from * 2 * part_floats;
        ca_join<DH, ROWS>(p, it, team_of(min(it.to, c1) - 1) - from + 1, [&](int j) { return base + (size_t)j * 2 * part_floats + (j == 0 && slot1 ? part_floats : 0); }, to,
                          member * 32 + lane, team_warps * 32);
    };
    float *cta_part = p.cta_parts + (size_t)blockIdx.x * 2 * part_floats;
    if (team == 0 && first_item_of_cta.from < c0) join_here(first_item_of_cta, 0, false, cta_part);
    const CaItem it = last_item_of[team];
    if (it.from >= u0 && it.to > u1) {  // begins in this team's share and goes on
        const bool goes_on = it.to > c1, slot1 = it.from > c0;
        join_here(it, team, it.from > u0, goes_on ? cta_part + (slot1 ? part_floats : 0) : nullptr);
        if (goes_on && leads && lane == 0) {
            p.items[2 * blockIdx.x] = make_int4(slot1 ? 2 : 1, ca_share_of(total, it.to - 1, ctas), it.head, it.tile);
            p.items[2 * blockIdx.x + 1] = make_int4(it.row0, it.m, 0, 0);
        }
    }
}

// Joins the parts of the items that several CTAs shared: block w the one that begins in CTA w's share and does not end there, if there is one; eight rows
// each.  A single row's parts, which can be as many as there are CTAs, are dealt to eight groups of threads.  ROWS_BESIDE: of a part sixteen bytes of each row, then
// the next sixteen of each (the tcgen05 form), else row after row.
template <int DH, int ROWS, bool ROWS_BESIDE>
__global__ void __launch_bounds__(8 * DH / 4) cached_attention_join_kernel(CaParams p) {
    constexpr int PART = 4 + 2 * DH, FOURS = DH / 4;
    __shared__ __align__(16) float smem[ROWS == 1 ? 8 * PART : 4];
    const int w0 = blockIdx.x, group = ROWS_BESIDE ? threadIdx.x % 8 : threadIdx.x / FOURS, dim = (ROWS_BESIDE ? threadIdx.x / 8 : threadIdx.x % FOURS) * 4, all = ROWS * p.tiles, part_floats = all * PART;
    pdl_wait();
    const int4 item = p.items[2 * w0], at = p.items[2 * w0 + 1];
    if (!item.x) return;
    const CaItem it = {0, 0, at.x, at.y, item.z, item.w};
    const int r = ROWS == 1 ? 0 : 8 * blockIdx.y + group, n = item.y - w0 + 1;
    if (r >= it.m * p.group - it.tile * all) return;
    const float *base = p.cta_parts + (size_t)w0 * 2 * part_floats + r * (ROWS_BESIDE ? 4 : PART);
    CaSum sum;
#pragma unroll 4
    for (int j = ROWS == 1 ? group : 0; j < n; j += ROWS == 1 ? 8 : 1) sum.add_part(base + (size_t)j * 2 * part_floats + (j == 0 && item.x == 2 ? part_floats : 0), DH, dim, ROWS_BESIDE ? all : 1);
    if (ROWS == 1) {
        sum.store_part(smem + group * PART, DH, dim, dim == 0);
        __syncthreads();
        if (group) return;
        sum = CaSum();
        for (int j = 0; j < min(n, 8); ++j) sum.add_part(smem + j * PART, DH, dim);
    }
    sum.write(p, it, it.tile * all + r, DH, dim);
}

// How a call's rows are dealt.  One row an item where they are single tokens with heads of their own, else tiles of eight rows where the sequences have up
// to that many on average, else of sixteen, two to a team where they have more than that, of 128 where they have more than 80 (any call is right
// in any of these forms; the sequences' lengths are on the device).  The output's type has no say, so that it says nothing but how the output is rounded.
struct CaForm {
    int rows, tiles, teams, stages, threads;
};
static CaForm ca_form(const hgf_cache *cache, int64_t n_seqs, int64_t n_rows, int n_heads) {
    const bool narrow = cache->head_dim == 64;
    const int group = n_heads / cache->n_heads;
    // (256 rows of 6000 tokens, 2 sequences, 16 heads of 64: 91 us here, 157 in tiles of sixteen; but 64 rows of 4096 tokens,
    // 16 heads of 128, 71 and 58, since half of a tile of 128 is empty.  Sequences of a page or less each go either way: 121 of up to 80 tokens, 60 rows of four heads a
    // K/V head, 389 here and 302 in tiles of sixteen; 100 of up to 63 tokens, 30 rows of eight heads, 80 and 119.  What would tell them apart is on the device.)
    if (n_rows * group > 80 * n_seqs) return CaForm{16, kCtRows / 16, 1, 0, kCtThreads};
    if (n_rows * group <= n_seqs) return narrow ? CaForm{1, 1, 8, 2, 256} : CaForm{1, 1, 4, 2, 128};
    if (n_rows * group <= 8 * n_seqs) return narrow ? CaForm{8, 1, 4, 4, 256} : CaForm{8, 1, 4, 2, 256};
    const int tiles = n_rows * group <= 16 * n_seqs ? 1 : 2, teams = 4 / tiles;
    return CaForm{16, tiles, teams, (narrow ? 16 : 8) / teams, 256};
}

// `kernel` and the joining of its parts, which are of tiles of p.tiles * ROWS rows.
template <int DH, int ROWS, bool ROWS_BESIDE>
static cudaError_t launch_with_join(void (*kernel)(CaParams), size_t smem, std::atomic<unsigned long long> &attr_done, const CaParams &p, int threads, cudaStream_t stream) {
    cudaError_t e = ensure_dynamic_smem(kernel, smem, attr_done);
    if (e != cudaSuccess) return e;
    const int sms = device_sm_count();
    if (!sms) return cudaErrorInvalidDevice;
    const int grid = sms < kCaMaxSms ? sms : kCaMaxSms;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cfg.stream = stream;
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    e = cudaLaunchKernelEx(&cfg, kernel, p);
    if (e != cudaSuccess) return e;
    cfg.dynamicSmemBytes = 0;
    cfg.gridDim = dim3((unsigned)grid, (unsigned)(ROWS == 16 ? 2 * p.tiles : 1));
    cfg.blockDim = dim3(8 * DH / 4);
    e = cudaLaunchKernelEx(&cfg, cached_attention_join_kernel<DH, ROWS, ROWS_BESIDE>, p);
    if (e != cudaSuccess) return e;
    count_launch(2);
    return cudaSuccess;
}
template <int DH, int ROWS>
static cudaError_t launch_cached_attention(const CaParams &p, int threads, cudaStream_t stream) {
    using C = CaCfg<DH, ROWS>;
    static_assert(C::SMEM <= 226 * 1024, "shared memory of a CTA");
    static std::atomic<unsigned long long> attr_done{0};
    return launch_with_join<DH, ROWS, false>(cached_attention_kernel<DH, ROWS>, C::SMEM, attr_done, p, threads, stream);
}
template <int DH>
static cudaError_t launch_cached_attention_tc(const CaParams &p, int threads, cudaStream_t stream) {
    static std::atomic<unsigned long long> attr_done{0};
    return launch_with_join<DH, 16, true>(cached_attention_tc_kernel<DH>, CtCfg<DH>::SMEM, attr_done, p, threads, stream);
}

static size_t ca_items_bytes() { return align_up((size_t)kCaMaxSms * 2 * sizeof(int4), 256); }
static size_t ca_cta_parts_bytes(int head_dim, const CaForm &f) { return align_up((size_t)kCaMaxSms * 2 * f.tiles * f.rows * (4 + 2 * head_dim) * 4, 256); }
static size_t ca_workspace(int head_dim, const CaForm &f) {
    return ca_items_bytes() + ca_cta_parts_bytes(head_dim, f) + (f.rows == 1 || !f.stages ? 0 : align_up((size_t)kCaMaxSms * f.teams * 2 * f.tiles * f.rows * (4 + 2 * head_dim) * 4, 256));
}

}  // namespace hgf

using namespace hgf;

extern "C" size_t hgf_cached_workspace_bytes(const hgf_cache *cache, int64_t n_seqs, int64_t n_rows, int32_t n_heads) {
    if (!cache || (cache->head_dim != 64 && cache->head_dim != 128) || cache->n_heads <= 0 || n_heads <= 0 || n_rows <= 0 || n_seqs <= 0) return 256;
    return ca_workspace(cache->head_dim, ca_form(cache, n_seqs, n_rows, n_heads));
}

extern "C" hgf_status hgf_diff_attention_cached(const hgf_cache *cache, const void *q, int64_t n_rows, int32_t n_heads, const int32_t *slots,
                                                const int32_t *starts, int64_t n_seqs, float lambda, float out_scale, void *out, void *workspace,
                                                size_t workspace_bytes, uint32_t flags, void *stream_) {
    if (!q || !slots || !starts || !out || n_rows <= 0 || n_heads <= 0 || (flags & ~HGF_FLAG_OUT_BF16)) return HGF_ERR_INVALID_ARG;
    CaParams p = {};
    if (const hgf_status st = parse_cache(cache, n_seqs, &p.c)) return st;
    if (n_heads % cache->n_heads || n_heads > 65535 || n_rows > (1 << 24) || n_rows * (n_heads / cache->n_heads) > 0x3fffffffll) return HGF_ERR_UNSUPPORTED_SHAPE;
    if (((uintptr_t)q | (uintptr_t)out) & 15u) return HGF_ERR_MISALIGNED;
    const int group = n_heads / cache->n_heads, dh = cache->head_dim;
    const CaForm f = ca_form(cache, n_seqs, n_rows, n_heads);
    if (!workspace || workspace_bytes < ca_workspace(dh, f)) return HGF_ERR_WORKSPACE;
    if ((uintptr_t)workspace & 255u) return HGF_ERR_MISALIGNED;
    p.q = (const __nv_bfloat16 *)q;
    p.slots = slots;
    p.starts = starts;
    p.out = out;
    p.items = (int4 *)workspace;
    p.cta_parts = (float *)((char *)workspace + ca_items_bytes());
    p.parts = (float *)((char *)p.cta_parts + ca_cta_parts_bytes(dh, f));
    p.status = device_status_word();
    if (!p.status) return HGF_ERR_CUDA;
    p.n_seqs = (int)n_seqs;
    p.n_rows = (int)n_rows;
    p.group = group;
    p.bf16 = (flags & HGF_FLAG_OUT_BF16) != 0;
    p.teams = f.teams;
    p.tiles = f.tiles;
    p.stages = f.stages;
    p.lambda = lambda;
    p.out_scale = out_scale;
    p.scale_log2 = (float)(1.4426950408889634 / sqrt((double)dh));
    p.per_group = (float)(1.0 / group);
    const cudaStream_t stream = (cudaStream_t)stream_;
    cudaError_t e;
    auto launch = [&](auto narrow, auto wide) { return (dh == 64 ? narrow : wide)(p, f.threads, stream); };
    if (!f.stages) e = launch(launch_cached_attention_tc<64>, launch_cached_attention_tc<128>);
    else if (f.rows == 1) e = launch(launch_cached_attention<64, 1>, launch_cached_attention<128, 1>);
    else if (f.rows == 8) e = launch(launch_cached_attention<64, 8>, launch_cached_attention<128, 8>);
    else e = launch(launch_cached_attention<64, 16>, launch_cached_attention<128, 16>);
    return e == cudaSuccess ? HGF_OK : HGF_ERR_CUDA;
}
