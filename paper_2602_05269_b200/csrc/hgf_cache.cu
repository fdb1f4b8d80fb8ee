// The 8-bit paged K/V cache of the differential attention: assigning and giving back pages, forking sequences, appending tokens (with the
// quantisation of the blocks that become complete) and reading them back.  The layout is in include/hgf.h; the attention over it in
// hgf_cached_attention.cu.
#include "hgf_cache.cuh"
#include "hgf_warp.cuh"

namespace hgf {

hgf_status parse_cache(const hgf_cache *c, int64_t n, CacheView *v) {
    if (!c || !c->codes || !c->scales || !c->open || !c->table || !c->held || !c->length || !c->refs || !c->arrivals) return HGF_ERR_INVALID_ARG;
    if (c->n_pages <= 0 || c->n_slots <= 0 || c->max_pages <= 0 || c->n_heads <= 0 || n <= 0) return HGF_ERR_INVALID_ARG;
    if ((c->head_dim != 64 && c->head_dim != 128) || c->n_heads > 65535 || c->n_pages > 0x7fffffffll || c->n_slots > 0x7fffffffll ||
        c->max_pages > (1 << 24) || n > kCacheMaxSeqs)
        return HGF_ERR_UNSUPPORTED_SHAPE;
    const uintptr_t all = (uintptr_t)c->codes | (uintptr_t)c->scales | (uintptr_t)c->open | (uintptr_t)c->table | (uintptr_t)c->held |
                          (uintptr_t)c->length | (uintptr_t)c->refs | (uintptr_t)c->arrivals;
    if (all & 15u) return HGF_ERR_MISALIGNED;
    v->codes = (int8_t *)c->codes;
    v->scales = (float4 *)c->scales;
    v->open = (__nv_bfloat16 *)c->open;
    v->table = c->table;
    v->held = c->held;
    v->length = c->length;
    v->refs = c->refs;
    v->arrivals = c->arrivals;
    v->n_pages = (int)c->n_pages;
    v->n_slots = (int)c->n_slots;
    v->max_pages = (int)c->max_pages;
    v->H = c->n_heads;
    return HGF_OK;
}

// One thread of each of `blocks` blocks calls this when its block has read all it needs of the slot's state: true for the last of them, which may
// change that state.  The counter is zero again afterwards.
__device__ static bool last_arrival(int32_t *arrivals, int blocks) {
    __threadfence();
    if (atomicAdd(arrivals, 1) != blocks - 1) return false;
    *arrivals = 0;
    __threadfence();
    return true;
}

// The sequence and piece of a block of threads: piece x of the launch belongs to sequence i, where sequence i has its pieces from
// starts[i] / 64 + i * per on (`per` pieces and one for each 64 rows are room for all that it can have).  All threads call it; `slots` (shared memory)
// holds the list of slots afterwards.
struct CachePiece {
    int i;        // -1: the starts are no ascending row numbers up to n_rows; -2: nobody's (before the first sequence's rows)
    int row0, m;  // the sequence's rows
    int piece, pieces;  // this one, and how many the sequence has in the launch, needed or not
    int slot;
    bool first;   // no earlier entry of the list names the slot
};
__device__ __forceinline__ CachePiece find_piece(const int32_t *__restrict__ list, const int32_t *__restrict__ starts, int n, int n_rows, int per, int x, int *slots) {
    CachePiece p = {-1, 0, 0, 0, 0, -1, false};
    int below = 0;
    bool bad = false;
    for (int j0 = 0; j0 < n; j0 += blockDim.x) {
        const int j = j0 + threadIdx.x;
        bool mine = false;
        if (j < n) {
            const int a = starts[j], b = starts[j + 1];
            slots[j] = list[j];
            bad = bad || a < 0 || b < a || b > n_rows;
            mine = (a >> 6) + j * per <= x;
        }
        below += __syncthreads_count(mine);
    }
    if (__syncthreads_or(bad)) return p;
    p.i = below ? below - 1 : -2;
    if (p.i < 0) return p;
    p.row0 = starts[p.i];
    p.m = starts[p.i + 1] - p.row0;
    p.piece = x - ((p.row0 >> 6) + p.i * per);
    p.pieces = (p.i + 1 < n ? ((p.row0 + p.m) >> 6) + (p.i + 1) * per : (int)gridDim.x) - (x - p.piece);
    p.slot = slots[p.i];
    bool again = false;
    for (int j = threadIdx.x; j < p.i; j += blockDim.x) again = again || slots[j] == p.slot;
    p.first = !__syncthreads_or(again);
    return p;
}
// Blocks of threads a piece's heads are dealt to, so that there are about `blocks` in all: a block's look-ups serve several heads where there are many pieces.
static unsigned head_shares(int64_t pieces, int H, int blocks) {
    const int64_t want = (blocks + pieces - 1) / pieces;
    const int64_t each = (H + (want < H ? want : H) - 1) / (want < H ? want : H);  // heads of a block
    return (unsigned)((H + each - 1) / each);
}

// ---- append ---------------------------------------------------------------------------------------------------------------------
// A block of threads takes one piece and every gridDim.y-th K/V head of it: a block of 64 tokens that becomes complete, whose values it reads from the open
// rows and the new ones, quantises, and writes as a page; the sequence's first piece also writes the rows that stay open, after its reads of the rows
// that these replace.  Each new value is read once, each code written once.  What bounds it is the chain of dependent look-ups in front (starts, slot, length,
// table, counts: about 4 us), which is why a block has several heads, and then that a block goes through its two or three heads in turn - reduce, barrier, quantise, barrier,
// store, the next head's loads under the stores - with all blocks in step.  Measured, kernel alone, memory cold: 64 sequences with one token each, 16 heads of 64, 10.6 us (the few whose
// block becomes complete end last); six with up to 1400 tokens 20.3 us for 53 MB (addresses found anew for every page 31).
constexpr int kAppendThreads = 256;

// Four lanes (l, l + 8, l + 16, l + 24) hold a word of four bytes each, a 4 x 4 matrix: its transpose.
__device__ __forceinline__ uint32_t transpose_bytes(uint32_t w, int lane) {
    uint32_t o = __shfl_xor_sync(0xffffffffu, w, 16);
    w = lane & 16 ? __byte_perm(o, w, 0x7632) : __byte_perm(w, o, 0x5410);
    o = __shfl_xor_sync(0xffffffffu, w, 8);
    return lane & 8 ? __byte_perm(o, w, 0x7351) : __byte_perm(w, o, 0x6240);
}

// Factor f with which rint(x f) is the rounding of the exact quotient 127 x / gamma, ties to even, for bf16 |x| <= gamma, in one multiplication.  With
// eight-bit mantissas X and G the quotient is 127 X 2^e / G; unless it is half-way between two integers it is 1 / (2 G) or more away from that, far more
// than two steps of f move it.  127 is a prime, so it is half-way only where 127 divides G, G = 254, or where it divides the odd number 2 n + 1 <= 254 of
// the point n + 1/2, so n = 63 and |x| = gamma / 2.  For G = 254 the factor is a power of two, the product exact and the tie left to the rounding; else the
// factor is the quotient 127 / gamma rounded and one step more, which takes |x| = gamma / 2 above 63.5, to the even 64.
__device__ __forceinline__ float code_factor(float gamma) {
    const float f = __fdiv_rn(127.0f, gamma);
    return (__float_as_uint(gamma) >> 16 & 0x7fu) == 0x7eu ? f : __uint_as_float(__float_as_uint(f) + 1u);
}
// Codes of eight values (two words), x * up * f: rounded by adding 1.5 * 2^23, whose low byte is then the code.
__device__ __forceinline__ uint2 codes8(const uint4 &v, float up, float f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    const uint64_t f2 = pack_f32x2(f, f), up2 = pack_f32x2(up, up), magic = pack_f32x2(12582912.0f, 12582912.0f);
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint64_t x = pack_f32x2(bf16lo_to_float(w[e]), bf16hi_to_float(w[e]));
        if (up != 1.0f) x = mul_f32x2(x, up2);
        float t0, t1;
        unpack_f32x2(fma_f32x2(x, f2, magic), t0, t1);
        b[2 * e] = __float_as_uint(t0);
        b[2 * e + 1] = __float_as_uint(t1);
    }
    uint32_t o[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) o[h] = __byte_perm(__byte_perm(b[4 * h], b[4 * h + 1], 0x0040), __byte_perm(b[4 * h + 2], b[4 * h + 3], 0x0040), 0x5410);
    return make_uint2(o[0], o[1]);
}

template <int DH>
__global__ void __launch_bounds__(kAppendThreads, DH == 64 ? 4 : 2) cache_append_kernel(CacheView c, const __nv_bfloat16 *__restrict__ k, const __nv_bfloat16 *__restrict__ v, int n_rows,
                                                                       const int32_t *__restrict__ slots, const int32_t *__restrict__ starts, int n_seqs, int32_t *done,
                                                                       unsigned int *status) {
    constexpr int EIGHTS = DH / 8, PER = kCacheBlock * EIGHTS / kAppendThreads, WARPS = kAppendThreads / 32;  // eights of a row; eights of one tensor's block a thread holds
    __shared__ __align__(16) uint8_t page_smem[3 * kCacheBlock * DH];
    __shared__ uint32_t top_smem[3][WARPS];
    __shared__ int slot_smem[kCacheMaxSeqs];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, head0 = blockIdx.y, H = c.H;
    pdl_launch_dependents();
    pdl_wait();
    const CachePiece p = find_piece(slots, starts, n_seqs, n_rows, 1, blockIdx.x, slot_smem);
    if (p.i < 0) {
        if (tid == 0 && p.i == -1) {
            atomicOr(status, kStatusCache);
            if (done && head0 == 0)
                for (int j = blockIdx.x; j < n_seqs; j += gridDim.x) done[j] = 0;
        }
        return;
    }
    const int i = p.i, row0 = p.row0, m = p.m, piece = p.piece, slot = p.slot;
    const bool leads = piece == 0 && head0 == 0 && tid == 0;
    if (slot < 0 || slot >= c.n_slots || !p.first) {
        if (leads) {
            if (done) done[i] = 0;
            if (slot != -1 && p.first) atomicOr(status, kStatusCache);
        }
        return;
    }
    const int held = c.held[slot], length = c.length[slot], block0 = length >> 6, open0 = length & 63;
    const long long after = (long long)length + m;
    const bool sane = cache_slot_ok(c, held, length);
    bool fits = sane && (after >> 6) <= held;
    const int blocks = fits ? (int)(after >> 6) - block0 : 0;
    const int32_t *table = c.table + (size_t)slot * c.max_pages + (sane ? block0 : 0);
    const size_t kw = (size_t)2 * H * DH, vw = (size_t)H * DH;
    auto open_rows = [&](int head) { return c.open + ((size_t)slot * H + head) * (3 * kCacheBlock * DH); };
    auto new_eight = [&](int n, int head, int row, int eight) {  // eight `eight` of a head of tensor n of the call's row `row`
        const __nv_bfloat16 *src = n < 2 ? k + (size_t)row * kw + ((size_t)n * H + head) * DH : v + (size_t)row * vw + (size_t)head * DH;
        return *reinterpret_cast<const uint4 *>(src + 8 * eight);
    };
    // A warp's lanes take eight eights of four rows; a thread's u-th unit lies ROWS_ON rows further down, at the same dims.
    constexpr int ROWS_ON = DH == 64 ? 32 : 16;
    const int r_first = DH == 64 ? 4 * warp + (lane >> 3) : 4 * (warp >> 1) + (lane >> 3), eight = DH == 64 ? lane & 7 : (warp & 1) * 8 + (lane & 7);
    const int t0 = (block0 + piece) * kCacheBlock;  // first token of the block
    uint4 x[3][PER];
    auto load = [&](int head) {
        const __nv_bfloat16 *open = open_rows(head);
        const __nv_bfloat16 *kp = k + (ptrdiff_t)(row0 + t0 + r_first - length) * (ptrdiff_t)kw + (size_t)head * DH + 8 * eight;  // (looked at from the first new row on)
        const __nv_bfloat16 *vp = v + (ptrdiff_t)(row0 + t0 + r_first - length) * (ptrdiff_t)vw + (size_t)head * DH + 8 * eight;
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int r = r_first + u * ROWS_ON;
            if (t0 + r < length) {
#pragma unroll
                for (int n = 0; n < 3; ++n) x[n][u] = *reinterpret_cast<const uint4 *>(open + ((size_t)n * kCacheBlock + r) * DH + 8 * cache_open_eight(r, eight));
            } else {
                x[0][u] = *reinterpret_cast<const uint4 *>(kp + (size_t)u * ROWS_ON * kw);
                x[1][u] = *reinterpret_cast<const uint4 *>(kp + (size_t)u * ROWS_ON * kw + vw);
                x[2][u] = *reinterpret_cast<const uint4 *>(vp + (size_t)u * ROWS_ON * vw);
            }
        }
    };
    // Where its bytes go in the page: of K the words of dims 0-3 and, sixteen bytes on, 4-7; of V, after four lanes' rows have become four bytes of a dim
    // each, the words of one of dims 0-3 and, 256 bytes on, one of dims 4-7.
    const int k_byte = cache_tile_byte(r_first, 8 * eight, DH), v_byte = cache_tile_byte(8 * eight + (lane >> 3), r_first & ~3, kCacheBlock);
    constexpr int K_ON = 2048;
    auto v_on = [](int u) { return DH == 64 ? 512 * u : 512 * (u >> 1) + 8 * (u & 1); };
    if (piece < blocks) load(head0);  // (on their way during the look-ups below)
    bool shared = false, off = false;
    for (int b = tid; b < blocks; b += kAppendThreads) {
        const int page = table[b];
        const bool ok = page >= 0 && page < c.n_pages;
        off = off || !ok;
        shared = shared || (ok && c.refs[page] != 1);
    }
    if (blocks) {
        off = __syncthreads_or(off);
        fits = !__syncthreads_or(shared) && !off;
    }
    if (!fits) {
        if (leads) {
            if (done) done[i] = 0;
            if (!sane || off) atomicOr(status, kStatusCache);
        }
        return;
    }

    // rows that stay open: those of the last block, or all new ones if none became complete
    auto keep_open = [&](int head) {
        constexpr int ROWS_AT_ONCE = kAppendThreads / EIGHTS;
        const int from = blocks ? 0 : open0, rows = blocks ? (int)(after & 63) : m, src0 = row0 + m - rows, e = tid % EIGHTS, r_mine = tid / EIGHTS;
#pragma unroll
        for (int q = 0; q < kCacheBlock / ROWS_AT_ONCE; ++q) {
            const int r = r_mine + q * ROWS_AT_ONCE;
            if (r < rows) {
                uint4 y[3];
#pragma unroll
                for (int n = 0; n < 3; ++n) y[n] = new_eight(n, head, src0 + r, e);
#pragma unroll
                for (int n = 0; n < 3; ++n) *reinterpret_cast<uint4 *>(open_rows(head) + ((size_t)n * kCacheBlock + from + r) * DH + 8 * cache_open_eight(from + r, e)) = y[n];
            }
        }
    };
    if (piece < blocks) {
        const int page = table[piece];
        for (int head = head0; head < H; head += gridDim.y) {
#pragma unroll
            for (int n = 0; n < 3; ++n) {
                uint32_t acc = 0;
#pragma unroll
                for (int u = 0; u < PER; ++u) acc = absmax8_bits(acc, x[n][u]);
                acc = __reduce_max_sync(0xffffffffu, max(acc >> 16, acc & 0xffffu));
                if (lane == 0) top_smem[n][warp] = acc;
            }
            __syncthreads();                  // (and the page before has left shared memory, and all of the block's open rows have been read)
            if (piece == 0) keep_open(head);
            uint32_t top[3];
#pragma unroll
            for (int n = 0; n < 3; ++n) {
                top[n] = 0;
#pragma unroll
                for (int w = 0; w < WARPS; ++w) top[n] = max(top[n], top_smem[n][w]);
                const float gamma = __uint_as_float(top[n] << 16);
                // (bf16 patterns from 0x7f80 on are infinities and NaN; below 2^-100 the factor could leave binary32's range)
                const bool zero = top[n] == 0 || top[n] >= 0x7f80u;
                const float up = gamma < 7.888609052210118e-31f ? 1.2676506002282294e30f : 1.0f, f = zero ? 0.0f : code_factor(gamma * up);
                uint8_t *dst = page_smem + n * kCacheBlock * DH + (n < 2 ? k_byte : v_byte);
#pragma unroll
                for (int u = 0; u < PER; ++u) {
                    const uint2 q = zero ? make_uint2(0, 0) : codes8(x[n][u], up, f);
                    if (n < 2) {
                        *reinterpret_cast<uint32_t *>(dst + u * K_ON) = q.x;
                        *reinterpret_cast<uint32_t *>(dst + u * K_ON + 16) = q.y;
                    } else {
                        *reinterpret_cast<uint32_t *>(dst + v_on(u)) = transpose_bytes(q.x, lane);
                        *reinterpret_cast<uint32_t *>(dst + v_on(u) + 256) = transpose_bytes(q.y, lane);
                    }
                }
            }
            if (head + gridDim.y < H) load(head + gridDim.y);
            __syncthreads();
            const size_t at = (size_t)page * H + head;
            uint4 *dst = reinterpret_cast<uint4 *>(c.codes + at * (3 * kCacheBlock * DH));
#pragma unroll
            for (int j = 0; j < 3 * kCacheBlock * DH / 16 / kAppendThreads; ++j) dst[tid + j * kAppendThreads] = reinterpret_cast<const uint4 *>(page_smem)[tid + j * kAppendThreads];
            if (tid == 0) {
                auto scale = [](uint32_t t) { return t >= 0x7f80u ? __uint_as_float(0x7fc00000u) : __fdiv_rn(__uint_as_float(t << 16), 127.0f); };
                c.scales[at] = make_float4(scale(top[0]), scale(top[1]), scale(top[2]), 0.0f);
            }
        }
    } else if (piece == 0) {
        for (int head = head0; head < H; head += gridDim.y) keep_open(head);
    }
    // (pieces that the sequence turned out not to need arrive as well: they have read its length, too)
    __syncthreads();
    if (tid == 0 && last_arrival(c.arrivals + slot, p.pieces * gridDim.y)) {
        c.length[slot] = (int)after;
        if (done) done[i] = 1;
    }
}

// ---- read -------------------------------------------------------------------------------------------------------------------------
// A block of threads takes one block of tokens that a range touches and every gridDim.y-th K/V head of it: the page through shared memory, whole, since a
// token's codes are spread over it, the next head's on its way meanwhile; open rows straight from where they are.  Bound by the writes: four sequences of up to
// 8192 tokens, 128 wide, fp32 out, 420 MB in all in 77 us, 83 % of the floor at 6567 GB/s of copy bandwidth (four bytes of output a thread and store: 97).
constexpr int kReadThreads = 256;

template <int DH>
constexpr int kReadSmem = 2 * 3 * kCacheBlock * DH;

__device__ __forceinline__ void copy_async16(uint32_t dst, const void *src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory"); }

// Byte k of w, a signed code, as a float.
__device__ __forceinline__ float code_float(uint32_t flipped, int k) { return __uint_as_float(__byte_perm(flipped, 0x4b000000u, 0x7540 + k)) - 8388736.0f; }

template <int DH, bool BF16>
__global__ void __launch_bounds__(kReadThreads, 4) cache_read_kernel(CacheView c, const int32_t *__restrict__ slots, const int32_t *__restrict__ firsts, const int32_t *__restrict__ starts,
                                                                   int n_seqs, int n_rows, void *__restrict__ k_out, void *__restrict__ v_out, unsigned int *status) {
    constexpr int EIGHTS = DH / 8, PAGE = 3 * kCacheBlock * DH;
    extern __shared__ __align__(16) uint8_t pages_smem[];
    __shared__ int slot_smem[kCacheMaxSeqs];
    const int tid = threadIdx.x, head0 = blockIdx.y, H = c.H;
    pdl_launch_dependents();
    pdl_wait();
    const CachePiece p = find_piece(slots, starts, n_seqs, n_rows, 2, blockIdx.x, slot_smem);
    if (p.i < 0) {
        if (tid == 0 && p.i == -1) atomicOr(status, kStatusCache);
        return;
    }
    const int row0 = p.row0, m = p.m, slot = p.slot;
    if (slot == -1 || m == 0) return;
    const int first = firsts[p.i];
    if (slot < 0 || slot >= c.n_slots || first < 0 || !cache_slot_ok(c, c.held[slot], c.length[slot])) {
        if (tid == 0) atomicOr(status, kStatusCache);
        return;
    }
    const int length = c.length[slot];
    const long long end = min((long long)first + m, (long long)length), b0 = (long long)((first >> 6) + p.piece) << 6;
    const int from = (int)max(b0, (long long)first), to = (int)min(b0 + kCacheBlock, end);
    if (from >= to) return;
    const int rows = to - from, r0 = (int)(from - b0);
    const size_t kw = (size_t)2 * H * DH, vw = (size_t)H * DH, out0 = (size_t)row0 + (from - first);
    auto put = [](void *base, size_t at, const auto &f) {
        constexpr int N = sizeof(f) / sizeof(float);
        if (BF16) {
            uint32_t w[N / 2];
#pragma unroll
            for (int b = 0; b < N / 2; ++b) {
                const __nv_bfloat162 x = __floats2bfloat162_rn(f[2 * b], f[2 * b + 1]);
                w[b] = *reinterpret_cast<const uint32_t *>(&x);
            }
            if constexpr (N == 8) *reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(base) + at) = make_uint4(w[0], w[1], w[2], w[3]);
            else *reinterpret_cast<uint2 *>(reinterpret_cast<__nv_bfloat16 *>(base) + at) = make_uint2(w[0], w[1]);
        } else {
#pragma unroll
            for (int b = 0; b < N; b += 4) *reinterpret_cast<float4 *>(reinterpret_cast<float *>(base) + at + b) = make_float4(f[b], f[b + 1], f[b + 2], f[b + 3]);
        }
    };
    // A thread has the same sixteen bytes of output of every ROWS_ON-th row of K1 or K2 in a page, and the same eight dims of every OPEN_ON-th open row.
    constexpr int DIMS = BF16 ? 8 : 4, UNITS = DH / DIMS, ROWS_ON = kReadThreads / (2 * UNITS), OPEN_ON = kReadThreads / EIGHTS;
    if (b0 + kCacheBlock > length) {
        const int e = tid % EIGHTS;
        for (int head = head0; head < H; head += gridDim.y)
#pragma unroll
            for (int q = 0; q < kCacheBlock / OPEN_ON; ++q) {
                const int r = tid / EIGHTS + q * OPEN_ON;
                if (r < r0 || r >= r0 + rows) continue;
                const __nv_bfloat16 *src = c.open + ((size_t)slot * H + head) * (3 * kCacheBlock * DH) + (size_t)r * DH + 8 * cache_open_eight(r, e);
                uint4 y[3];
#pragma unroll
                for (int n = 0; n < 3; ++n) y[n] = *reinterpret_cast<const uint4 *>(src + n * kCacheBlock * DH);
#pragma unroll
                for (int n = 0; n < 3; ++n) {
                    const size_t row = out0 + r - r0;
                    const size_t at = n < 2 ? row * kw + ((size_t)n * H + head) * DH + 8 * e : row * vw + (size_t)head * DH + 8 * e;
                    if (BF16) {
                        *reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(n < 2 ? k_out : v_out) + at) = y[n];
                    } else {
                        float f[8];
                        unpack8(y[n], f);
                        put(n < 2 ? k_out : v_out, at, f);
                    }
                }
            }
        return;
    }
    const int page = c.table[(size_t)slot * c.max_pages + (int)(b0 >> 6)];
    if (page < 0 || page >= c.n_pages) {
        if (tid == 0) atomicOr(status, kStatusCache);
        return;
    }
    const uint32_t smem = dsmem_u32(pages_smem);
    auto fetch = [&](int head, int buf) {
        if (head < H) {
            const int8_t *src = c.codes + ((size_t)page * H + head) * PAGE;
#pragma unroll
            for (int j = 0; j < PAGE / 16 / kReadThreads; ++j) copy_async16(smem + buf * PAGE + (tid + j * kReadThreads) * 16, src + (tid + j * kReadThreads) * 16);
        }
        asm volatile("cp.async.commit_group;\n" ::: "memory");
    };
    fetch(head0, 0);
    const int dim = tid % UNITS * DIMS, n = tid / UNITS & 1, r_first = tid / (2 * UNITS), d4 = tid % (DH / 4) * 4, r4 = tid / (DH / 4) * 4;
    const int k_byte = n * kCacheBlock * DH + cache_tile_byte(r_first, dim, DH), v_byte = 2 * kCacheBlock * DH + cache_tile_byte(d4, r4, kCacheBlock);
    int buf = 0;
    for (int head = head0; head < H; head += gridDim.y, buf ^= 1) {
        const float4 sc = c.scales[(size_t)page * H + head];
        fetch(head + gridDim.y, buf ^ 1);
        asm volatile("cp.async.wait_group 1;\n" ::: "memory");
        __syncthreads();
        const uint8_t *src = pages_smem + buf * PAGE;
        const float s = n ? sc.y : sc.x;
        const size_t k_at = ((ptrdiff_t)out0 - r0 + r_first) * (ptrdiff_t)kw + ((size_t)n * H + head) * DH + dim;
#pragma unroll
        for (int q = 0; q < kCacheBlock / ROWS_ON; ++q) {
            const int r = r_first + q * ROWS_ON;
            if (r < r0 || r >= r0 + rows) continue;
            const uint8_t *at = src + k_byte + cache_tile_byte(q * ROWS_ON, 0, DH);  // (r_first and the step have no bit in common)
            float f[DIMS];
#pragma unroll
            for (int h = 0; h < DIMS / 4; ++h) {
                const uint32_t w = *reinterpret_cast<const uint32_t *>(at + 16 * h) ^ 0x80808080u;
#pragma unroll
                for (int b = 0; b < 4; ++b) f[4 * h + b] = code_float(w, b) * s;
            }
            put(k_out, k_at + (size_t)q * ROWS_ON * kw, f);
        }
        // four rows of four dims of V at a time: a word is four tokens of a dim, and the next dim's is 64 bytes on
#pragma unroll
        for (int u = 0; u < DH / 64; ++u) {
            const int row = r4 + 32 * u;
            if (row + 3 < r0 || row >= r0 + rows) continue;
            uint32_t w[4];
#pragma unroll
            for (int b = 0; b < 4; ++b) w[b] = *reinterpret_cast<const uint32_t *>(src + v_byte + u * 512 + b * 64) ^ 0x80808080u;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float f[4] = {code_float(w[0], r) * sc.z, code_float(w[1], r) * sc.z, code_float(w[2], r) * sc.z, code_float(w[3], r) * sc.z};
                if (row + r >= r0 && row + r < r0 + rows) put(v_out, (out0 + row + r - r0) * vw + (size_t)head * DH + d4, f);
            }
        }
        __syncthreads();
    }
}

// ---- pages ------------------------------------------------------------------------------------------------------------------------
// Exclusive sum over the block's threads (1024), and the sum of all.
__device__ static int block_exclusive_sum(int v, int *smem /* [32] */, int *total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += t;
    }
    __syncthreads();
    if (lane == 31) smem[warp] = s;
    __syncthreads();
    int w = smem[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += t;
    }
    *total = __shfl_sync(0xffffffffu, w, 31);
    const int before = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
    return s - v + (warp ? before : 0);
}

// One block of threads deals the lowest free pages: the requests' running sum of pages in shared memory, then the reference counts in order, each free
// page to the request that its rank falls into.  A first walk counts the free pages, as far as they are asked for, so that a request that cannot be
// met in full takes none.  Bound by its dependent look-ups: 6.9 us for one request, 10.5 for 48 sequences of up to 4000 tokens.
constexpr int kReserveThreads = 1024, kReserveStep = 16;  // reference counts a thread looks at in one step

__global__ void __launch_bounds__(kReserveThreads) cache_reserve_kernel(CacheView c, const int32_t *__restrict__ slots, const int32_t *__restrict__ tokens, int n, int32_t *granted,
                                                                        unsigned int *status) {
    __shared__ __align__(16) int slot_of[kCacheMaxSeqs];
    __shared__ int upto[kCacheMaxSeqs], held_of[kCacheMaxSeqs], sums[32];
    __shared__ long long wide[32];
    __shared__ int dealt_smem;
    const int tid = threadIdx.x;
    pdl_launch_dependents();
    pdl_wait();
    const int slot = tid < n ? slots[tid] : -1;
    slot_of[tid] = slot;
    if (tid == 0) dealt_smem = 0;
    __syncthreads();
    bool able = tid < n && slot != -1;
    if (able && (slot < 0 || slot >= c.n_slots)) {
        atomicOr(status, kStatusCache);
        able = false;
    }
    int need = 0, held = able ? c.held[slot] : 0;
    const int want = able ? tokens[tid] : 0;
#pragma unroll 4
    for (int j = 0; able && j + 4 <= tid; j += 4) {
        const int4 v = *reinterpret_cast<const int4 *>(slot_of + j);
        able = able && v.x != slot && v.y != slot && v.z != slot && v.w != slot;
    }
    for (int j = tid & ~3; able && j < tid; ++j) able = slot_of[j] != slot;
    if (able) {
        if (held < 0 || held > c.max_pages || want < 0) {
            atomicOr(status, kStatusCache);
            able = false;
        } else if ((want >> 6) > c.max_pages) {
            able = false;
        } else {
            need = max(0, (want >> 6) - held);
        }
    }
    // (the sum saturates: n * 2^24 can pass 32 bits, the pool cannot)
    int total;
    {
        long long s = need;
        const int lane = tid & 31, warp = tid >> 5;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long t = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += t;
        }
        if (lane == 31) wide[warp] = s;
        __syncthreads();
        long long w = wide[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long t = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += t;
        }
        const long long all = __shfl_sync(0xffffffffu, w, 31), upto_here = __shfl_sync(0xffffffffu, w, (warp + 31) & 31), before = warp ? upto_here : 0;
        upto[tid] = (int)min(s + before, 0x7fffffffll);
        held_of[tid] = held;
        total = (int)min(all, 0x7fffffffll);
    }
    __syncthreads();
    constexpr int STEP = kReserveThreads * kReserveStep;
    auto free_pages = [&](long long p0) {  // of this thread's sixteen from p0 on: a bit each
        uint32_t mask = 0;
        const long long at = p0 + tid * kReserveStep;
        if (at + kReserveStep <= c.n_pages) {
            int4 v[kReserveStep / 4];
#pragma unroll
            for (int u = 0; u < kReserveStep / 4; ++u) v[u] = *reinterpret_cast<const int4 *>(c.refs + at + 4 * u);
#pragma unroll
            for (int u = 0; u < kReserveStep / 4; ++u)
                mask |= ((v[u].x == 0 ? 1u : 0u) | (v[u].y == 0 ? 2u : 0u) | (v[u].z == 0 ? 4u : 0u) | (v[u].w == 0 ? 8u : 0u)) << (4 * u);
        } else {
            int v[kReserveStep];
#pragma unroll
            for (int u = 0; u < kReserveStep; ++u) v[u] = at + u < c.n_pages ? c.refs[at + u] : 1;
#pragma unroll
            for (int u = 0; u < kReserveStep; ++u) mask |= (v[u] == 0 ? 1u : 0u) << u;
        }
        return mask;
    };
    constexpr int KEPT = 4;  // steps whose pages the second walk has at hand
    uint32_t kept[KEPT] = {};
    int found = 0;
    if (total > 0) {
        int step = 0;
        for (long long p0 = 0; p0 < c.n_pages && found < total; p0 += STEP, ++step) {
            const uint32_t mask = free_pages(p0);
#pragma unroll
            for (int u = 0; u < KEPT; ++u)
                if (u == step) kept[u] = mask;
            int sum;
            block_exclusive_sum(__popc(mask), sums, &sum);
            found += sum;
        }
    }
    const bool met = able && (need == 0 || upto[tid] <= found);
    if (granted && tid < n) granted[tid] = met;
    // pages dealt: as far as the requests that are met reach
    if (met && need) atomicMax(&dealt_smem, upto[tid]);
    __syncthreads();
    const int dealt = dealt_smem;
    int base = 0;
    int step = 0;
    for (long long p0 = 0; p0 < c.n_pages && base < dealt; p0 += STEP, ++step) {
        uint32_t free_mask = kept[0];
#pragma unroll
        for (int u = 1; u < KEPT; ++u)
            if (u == step) free_mask = kept[u];
        if (step >= KEPT) free_mask = free_pages(p0);
        int sum, rank = base + block_exclusive_sum(__popc(free_mask), sums, &sum);
        base += sum;
        if (free_mask && rank < dealt) {
            int lo = 0, hi = n - 1;  // the first request whose running sum is above the rank
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (upto[mid] > rank) hi = mid; else lo = mid + 1;
            }
            int32_t *entry = nullptr;  // where the rank's page goes
            for (int end = 0; free_mask && rank < dealt; free_mask &= free_mask - 1, ++rank, ++entry) {
                if (rank >= end) {
                    while (upto[lo] <= rank) ++lo;
                    end = upto[lo];
                    entry = c.table + (size_t)slot_of[lo] * c.max_pages + held_of[lo] + rank - (lo ? upto[lo - 1] : 0);
                }
                const int p = (int)(p0 + tid * kReserveStep + __ffs(free_mask) - 1);
                *entry = p;
                c.refs[p] = 1;
            }
        }
    }
    if (met && need) c.held[slot] = held + need;
}

__global__ void __launch_bounds__(256) cache_free_kernel(CacheView c, const int32_t *__restrict__ slots, unsigned int *status) {
    pdl_launch_dependents();
    pdl_wait();
    const int i = blockIdx.x, slot = slots[i];
    const bool first = cache_first_of(slots, i, slot);
    if (slot == -1 || !first) return;
    bool off = slot < 0 || slot >= c.n_slots;
    if (!off) {
        const int held = c.held[slot];
        off = held < 0 || held > c.max_pages;
        if (!off)
            for (int b = threadIdx.x; b < held; b += blockDim.x) {
                const int page = c.table[(size_t)slot * c.max_pages + b];
                if (page < 0 || page >= c.n_pages) {
                    off = true;
                } else if (atomicSub(c.refs + page, 1) <= 0) {  // (nobody held it)
                    atomicAdd(c.refs + page, 1);
                    off = true;
                }
            }
        __syncthreads();  // every thread has read `held`
        if (threadIdx.x == 0) {
            c.held[slot] = 0;
            c.length[slot] = 0;
        }
    }
    if (off) atomicOr(status, kStatusCache);
}

// A block of threads copies the open rows of every gridDim.y-th K/V head; the first of a pair also shares the pages, and the last to have read the state
// changes it.  Bound by the copy, 11.2 us for 144 forks (7 for three): the rows are asked for before it is known whether the copy is made.
template <int DH>
__global__ void __launch_bounds__(256) cache_fork_kernel(CacheView c, const int32_t *__restrict__ srcs, const int32_t *__restrict__ dsts, int n, int32_t *done, unsigned int *status) {
    const int i = blockIdx.x, head0 = blockIdx.y, tid = threadIdx.x, H = c.H;
    pdl_launch_dependents();
    pdl_wait();
    const int src = srcs[i], dst = dsts[i];
    const bool skip = src == -1 || dst == -1, off = !skip && (src < 0 || src >= c.n_slots || dst < 0 || dst >= c.n_slots), look = !skip && !off;
    const int held = look ? c.held[src] : 0, length = look ? c.length[src] : 0;
    bool empty = look && c.held[dst] == 0 && c.length[dst] == 0;
    const bool sane = look && cache_slot_ok(c, held, length);
    bool clash = false;
    for (int j = tid; j < n; j += blockDim.x) clash = clash || (j < i && dsts[j] == dst) || dsts[j] == src;
    const int full = sane ? length >> 6 : 0, rows = sane ? length & 63 : 0;
    bool bad_page = false;
    if (look)
        for (int b = tid; b < full; b += blockDim.x) {
            const int page = c.table[(size_t)src * c.max_pages + b];
            bad_page = bad_page || page < 0 || page >= c.n_pages;
        }
    // `per` units of sixteen bytes of each of the three of each head: six of these parts at a time, a unit of each in flight per thread
    const int per = rows * (DH / 8), parts = (H - head0 + gridDim.y - 1) / gridDim.y * 3;
    constexpr int AT_ONCE = 6, TENSOR = kCacheBlock * DH / 8;
    const uint4 *from = reinterpret_cast<const uint4 *>(c.open) + ((size_t)(look ? src : 0) * H + head0) * (3 * TENSOR);
    uint4 *to = reinterpret_cast<uint4 *>(c.open) + ((size_t)(look ? dst : 0) * H + head0) * (3 * TENSOR);
    uint4 v[AT_ONCE];
    auto load = [&](int part0, int at) {
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
            if (part0 + u < parts && at < per) v[u] = from[((size_t)((part0 + u) / 3) * gridDim.y * 3 + (part0 + u) % 3) * TENSOR + at];
    };
    load(0, tid);
    clash = __syncthreads_or(clash);
    bad_page = __syncthreads_or(bad_page);
    empty = empty && !clash;
    if (!empty || !sane || bad_page) {
        if (head0 == 0 && tid == 0) {
            if (done) done[i] = 0;
            if (off || (empty && !sane) || bad_page) atomicOr(status, kStatusCache);
        }
        return;
    }
    for (int part0 = 0; part0 < parts; part0 += AT_ONCE)
        for (int at = tid; at < per; at += 256) {
            if (part0 || at != tid) load(part0, at);
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (part0 + u < parts) to[((size_t)((part0 + u) / 3) * gridDim.y * 3 + (part0 + u) % 3) * TENSOR + at] = v[u];
        }
    if (head0 == 0)
        for (int b = tid; b < full; b += blockDim.x) {
            const int page = c.table[(size_t)src * c.max_pages + b];
            c.table[(size_t)dst * c.max_pages + b] = page;
            atomicAdd(c.refs + page, 1);
        }
    __syncthreads();
    if (tid == 0 && last_arrival(c.arrivals + dst, gridDim.y)) {
        c.held[dst] = full;
        c.length[dst] = length;
        if (done) done[i] = 1;
    }
}

// Launches with the attribute that lets a kernel's blocks start, up to their wait for the kernel before, while that one still runs.
template <class... A, class... B>
static hgf_status launch(void (*kernel)(A...), dim3 grid, int threads, size_t smem, void *stream, B... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, A(args)...) != cudaSuccess) return HGF_ERR_CUDA;
    count_launch();
    return HGF_OK;
}

}  // namespace hgf

using namespace hgf;

extern "C" hgf_status hgf_cache_reserve(const hgf_cache *cache, const int32_t *slots, const int32_t *tokens, int64_t n, int32_t *granted, void *stream) {
    CacheView c;
    if (!slots || !tokens) return HGF_ERR_INVALID_ARG;
    if (const hgf_status st = parse_cache(cache, n, &c)) return st;
    unsigned int *status = device_status_word();
    if (!status) return HGF_ERR_CUDA;
    return launch(cache_reserve_kernel, dim3(1), kReserveThreads, 0, stream, c, slots, tokens, (int)n, granted, status);
}

extern "C" hgf_status hgf_cache_append(const hgf_cache *cache, const void *k, const void *v, int64_t n_rows, const int32_t *slots, const int32_t *starts,
                                       int64_t n_seqs, int32_t *done, void *stream) {
    CacheView c;
    if (!k || !v || !slots || !starts || n_rows <= 0) return HGF_ERR_INVALID_ARG;
    if (const hgf_status st = parse_cache(cache, n_seqs, &c)) return st;
    if (n_rows > (1 << 24)) return HGF_ERR_UNSUPPORTED_SHAPE;
    if (((uintptr_t)k | (uintptr_t)v) & 15u) return HGF_ERR_MISALIGNED;
    unsigned int *status = device_status_word();
    if (!status) return HGF_ERR_CUDA;
    const int64_t pieces = n_rows / kCacheBlock + n_seqs;
    return launch(cache->head_dim == 64 ? cache_append_kernel<64> : cache_append_kernel<128>, dim3((unsigned)pieces, head_shares(pieces, c.H, 600)), kAppendThreads, 0, stream, c,
                  (const __nv_bfloat16 *)k, (const __nv_bfloat16 *)v, (int)n_rows, slots, starts, (int)n_seqs, done, status);
}

extern "C" hgf_status hgf_cache_read(const hgf_cache *cache, const int32_t *slots, const int32_t *first, const int32_t *starts, int64_t n_seqs, int64_t n_rows,
                                     void *k_out, void *v_out, uint32_t flags, void *stream) {
    CacheView c;
    if (!slots || !first || !starts || !k_out || !v_out || n_rows <= 0 || (flags & ~HGF_FLAG_OUT_BF16)) return HGF_ERR_INVALID_ARG;
    if (const hgf_status st = parse_cache(cache, n_seqs, &c)) return st;
    if (n_rows > (1 << 24)) return HGF_ERR_UNSUPPORTED_SHAPE;
    if (((uintptr_t)k_out | (uintptr_t)v_out) & 15u) return HGF_ERR_MISALIGNED;
    unsigned int *status = device_status_word();
    if (!status) return HGF_ERR_CUDA;
    const int64_t pieces = n_rows / kCacheBlock + 2 * n_seqs;
    const bool bf16 = (flags & HGF_FLAG_OUT_BF16) != 0, narrow = cache->head_dim == 64;
    auto kernel = narrow ? (bf16 ? cache_read_kernel<64, true> : cache_read_kernel<64, false>) : (bf16 ? cache_read_kernel<128, true> : cache_read_kernel<128, false>);
    static std::atomic<unsigned long long> done_wide{0}, done_wide_bf16{0};
    if (!narrow && ensure_dynamic_smem(kernel, kReadSmem<128>, bf16 ? done_wide_bf16 : done_wide) != cudaSuccess) return HGF_ERR_CUDA;
    return launch(kernel, dim3((unsigned)pieces, head_shares(pieces, c.H, 1600)), kReadThreads, narrow ? kReadSmem<64> : kReadSmem<128>, stream, c, slots, first, starts, (int)n_seqs,
                  (int)n_rows, k_out, v_out, status);
}

extern "C" hgf_status hgf_cache_fork(const hgf_cache *cache, const int32_t *src, const int32_t *dst, int64_t n, int32_t *done, void *stream) {
    CacheView c;
    if (!src || !dst) return HGF_ERR_INVALID_ARG;
    if (const hgf_status st = parse_cache(cache, n, &c)) return st;
    unsigned int *status = device_status_word();
    if (!status) return HGF_ERR_CUDA;
    return launch(cache->head_dim == 64 ? cache_fork_kernel<64> : cache_fork_kernel<128>, dim3((unsigned)n, head_shares(n, c.H, 600)), 256, 0, stream, c, src, dst, (int)n, done, status);
}

extern "C" hgf_status hgf_cache_free(const hgf_cache *cache, const int32_t *slots, int64_t n, void *stream) {
    CacheView c;
    if (!slots) return HGF_ERR_INVALID_ARG;
    if (const hgf_status st = parse_cache(cache, n, &c)) return st;
    unsigned int *status = device_status_word();
    if (!status) return HGF_ERR_CUDA;
    return launch(cache_free_kernel, dim3((unsigned)n), 256, 0, stream, c, slots, status);
}
