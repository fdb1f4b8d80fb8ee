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

// ---- append ---------------------------------------------------------------------------------------------------------------------
// A block of threads takes one K/V head of one piece: a block of 64 tokens that becomes complete, whose values it reads from the open rows and the
// new ones, quantises, and writes as a page; the sequence's first piece also writes the rows that stay open, after its reads of the rows that
// these replace.  Bound by memory: each new value is read once, each code written once.
constexpr int kAppendThreads = 256;

template <int DH>
__global__ void __launch_bounds__(kAppendThreads) cache_append_kernel(CacheView c, const __nv_bfloat16 *__restrict__ k, const __nv_bfloat16 *__restrict__ v, int n_rows,
                                                                       const int32_t *__restrict__ slots, const int32_t *__restrict__ starts, int n_seqs, int32_t *done,
                                                                       unsigned int *status) {
    constexpr int EIGHTS = DH / 8, PER = kCacheBlock * EIGHTS / kAppendThreads;  // eights of a row; eights of one tensor's block a thread holds
    __shared__ __align__(16) uint8_t page_smem[3 * kCacheBlock * DH];
    __shared__ uint32_t top_smem[3][kAppendThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, head = blockIdx.y, H = c.H;

    const int i = cache_find_sequence(starts, n_seqs, n_rows, 1, blockIdx.x);
    if (i < 0) {
        if (tid == 0) {
            atomicOr(status, kStatusCache);
            if (done && head == 0)
                for (int j = blockIdx.x; j < n_seqs; j += gridDim.x) done[j] = 0;
        }
        return;
    }
    const int row0 = starts[i], m = starts[i + 1] - row0, piece = (int)blockIdx.x - ((row0 >> 6) + i), slot = slots[i];
    const bool first = cache_first_of(slots, i, slot), leads = piece == 0 && head == 0 && tid == 0;
    if (slot < 0 || slot >= c.n_slots || !first) {
        if (leads) {
            if (done) done[i] = 0;
            if (slot != -1 && first) atomicOr(status, kStatusCache);
        }
        return;
    }
    const int held = c.held[slot], length = c.length[slot], block0 = length >> 6, open0 = length & 63;
    const long long after = (long long)length + m;
    const bool sane = cache_slot_ok(c, held, length);
    bool fits = sane && (after >> 6) <= held, in_range = true;
    const int blocks = fits ? (int)(after >> 6) - block0 : 0;
    const int32_t *table = c.table + (size_t)slot * c.max_pages + (sane ? block0 : 0);
    {
        bool shared = false, off = false;
        for (int b = tid; b < blocks; b += kAppendThreads) {
            const int page = table[b];
            const bool ok = page >= 0 && page < c.n_pages;
            off = off || !ok;
            shared = shared || (ok && c.refs[page] != 1);
        }
        in_range = !__syncthreads_or(off);
        fits = !__syncthreads_or(shared) && fits && in_range;
    }
    if (!fits) {
        if (leads) {
            if (done) done[i] = 0;
            if (!sane || !in_range) atomicOr(status, kStatusCache);
        }
        return;
    }
    const int pieces = blocks > 1 ? blocks : 1;
    if (piece >= pieces) return;

    const size_t kw = (size_t)2 * H * DH, vw = (size_t)H * DH;
    __nv_bfloat16 *open = c.open + ((size_t)slot * H + head) * (3 * kCacheBlock * DH);
    auto new_eight = [&](int n, int row, int eight) {  // eight `eight` of tensor n of the call's row `row`
        const __nv_bfloat16 *src = n < 2 ? k + (size_t)row * kw + ((size_t)n * H + head) * DH : v + (size_t)row * vw + (size_t)head * DH;
        return *reinterpret_cast<const uint4 *>(src + 8 * eight);
    };
    if (piece < blocks) {
        const int t0 = (block0 + piece) * kCacheBlock;  // first token of the block
        uint4 x[3][PER];
        uint32_t top[3];
#pragma unroll
        for (int n = 0; n < 3; ++n) {
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const int at = tid + u * kAppendThreads, r = at / EIGHTS, e = at % EIGHTS;
                x[n][u] = t0 + r < length ? *reinterpret_cast<const uint4 *>(open + ((size_t)n * kCacheBlock + r) * DH + 8 * cache_open_eight(r, e))
                                          : new_eight(n, row0 + t0 + r - length, e);
            }
        }
#pragma unroll
        for (int n = 0; n < 3; ++n) {
            uint32_t acc = 0;
#pragma unroll
            for (int u = 0; u < PER; ++u) acc = absmax8_bits(acc, x[n][u]);
            acc = __reduce_max_sync(0xffffffffu, max(acc >> 16, acc & 0xffffu));
            if (lane == 0) top_smem[n][warp] = acc;
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < 3; ++n) {
            top[n] = 0;
#pragma unroll
            for (int w = 0; w < kAppendThreads / 32; ++w) top[n] = max(top[n], top_smem[n][w]);
            const float gamma = __uint_as_float(top[n] << 16);
            // (bf16 patterns from 0x7f80 on are infinities and NaN; below 2^-100 the quotient 127 / max could leave binary32's range)
            const bool zero = top[n] == 0 || top[n] >= 0x7f80u;
            QuantScale s = make_quant_scale(gamma);
            if (gamma < 7.9e-31f) s.fast = false;
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const int at = tid + u * kAppendThreads, r = at / EIGHTS, e = at % EIGHTS;
                int sum = 0;
                const uint2 q = zero ? make_uint2(0, 0) : quant8(x[n][u], s, sum);
                if (n < 2) {
                    uint8_t *dst = page_smem + n * kCacheBlock * DH;
                    *reinterpret_cast<uint32_t *>(dst + cache_tile_byte(r, 8 * e, DH)) = q.x;
                    *reinterpret_cast<uint32_t *>(dst + cache_tile_byte(r, 8 * e + 4, DH)) = q.y;
                } else {
                    uint8_t *dst = page_smem + 2 * kCacheBlock * DH;
#pragma unroll
                    for (int b = 0; b < 8; ++b) dst[cache_tile_byte(8 * e + b, r, kCacheBlock)] = (uint8_t)((b < 4 ? q.x : q.y) >> (8 * (b & 3)));
                }
            }
        }
        __syncthreads();
        const size_t at = (size_t)table[piece] * H + head;
        uint4 *dst = reinterpret_cast<uint4 *>(c.codes + at * (3 * kCacheBlock * DH));
        for (int j = tid; j < 3 * kCacheBlock * DH / 16; j += kAppendThreads) dst[j] = reinterpret_cast<const uint4 *>(page_smem)[j];
        if (tid == 0) {
            auto scale = [](uint32_t t) { return t >= 0x7f80u ? __uint_as_float(0x7fc00000u) : __fdiv_rn(__uint_as_float(t << 16), 127.0f); };
            c.scales[at] = make_float4(scale(top[0]), scale(top[1]), scale(top[2]), 0.0f);
        }
    }
    if (piece == 0) {
        // rows that stay open: those of the last block, or all new ones if none became complete
        const int from = blocks ? 0 : open0, rows = blocks ? (int)(after & 63) : m, src0 = row0 + m - rows;
        for (int at = tid; at < 3 * rows * EIGHTS; at += kAppendThreads) {
            const int n = at / (rows * EIGHTS), r = at / EIGHTS % rows, e = at % EIGHTS;
            *reinterpret_cast<uint4 *>(open + ((size_t)n * kCacheBlock + from + r) * DH + 8 * cache_open_eight(from + r, e)) = new_eight(n, src0 + r, e);
        }
    }
    __syncthreads();
    if (tid == 0 && last_arrival(c.arrivals + slot, pieces * H)) {
        c.length[slot] = (int)after;
        if (done) done[i] = 1;
    }
}

// ---- read -------------------------------------------------------------------------------------------------------------------------
// A block of threads takes one K/V head of one block of tokens that a range touches: the page through shared memory, whole, since a token's codes are
// spread over it; open rows straight from where they are.
constexpr int kReadThreads = 256;

template <int DH, bool BF16>
__global__ void __launch_bounds__(kReadThreads) cache_read_kernel(CacheView c, const int32_t *__restrict__ slots, const int32_t *__restrict__ firsts, const int32_t *__restrict__ starts,
                                                                   int n_seqs, int n_rows, void *__restrict__ k_out, void *__restrict__ v_out, unsigned int *status) {
    constexpr int EIGHTS = DH / 8;
    __shared__ __align__(16) uint8_t page_smem[3 * kCacheBlock * DH];
    const int tid = threadIdx.x, head = blockIdx.y, H = c.H;
    const int i = cache_find_sequence(starts, n_seqs, n_rows, 2, blockIdx.x);
    if (i < 0) {
        if (tid == 0) atomicOr(status, kStatusCache);
        return;
    }
    const int row0 = starts[i], m = starts[i + 1] - row0, piece = (int)blockIdx.x - ((row0 >> 6) + 2 * i), slot = slots[i];
    if (slot == -1 || m == 0) return;
    const int first = firsts[i];
    if (slot < 0 || slot >= c.n_slots || first < 0 || !cache_slot_ok(c, c.held[slot], c.length[slot])) {
        if (tid == 0) atomicOr(status, kStatusCache);
        return;
    }
    const int length = c.length[slot];
    const long long end = min((long long)first + m, (long long)length), b0 = (long long)((first >> 6) + piece) << 6;
    const int from = (int)max(b0, (long long)first), to = (int)min(b0 + kCacheBlock, end);
    if (from >= to) return;
    const bool closed = b0 + kCacheBlock <= length;
    const __nv_bfloat16 *open = c.open + ((size_t)slot * H + head) * (3 * kCacheBlock * DH);
    float sc[3] = {0.0f, 0.0f, 0.0f};
    if (closed) {
        const int page = c.table[(size_t)slot * c.max_pages + (int)(b0 >> 6)];
        if (page < 0 || page >= c.n_pages) {
            if (tid == 0) atomicOr(status, kStatusCache);
            return;
        }
        const size_t at = (size_t)page * H + head;
        const uint4 *src = reinterpret_cast<const uint4 *>(c.codes + at * (3 * kCacheBlock * DH));
#pragma unroll 4
        for (int j = tid; j < 3 * kCacheBlock * DH / 16; j += kReadThreads) reinterpret_cast<uint4 *>(page_smem)[j] = src[j];
        const float4 s4 = c.scales[at];
        sc[0] = s4.x;
        sc[1] = s4.y;
        sc[2] = s4.z;
        __syncthreads();
    }
    const int rows = to - from, r0 = (int)(from - b0);
    const size_t kw = (size_t)2 * H * DH, vw = (size_t)H * DH, out0 = (size_t)row0 + (from - first);
#pragma unroll
    for (int n = 0; n < 3; ++n)
        for (int at = tid; at < rows * EIGHTS; at += kReadThreads) {
            const int r = r0 + at / EIGHTS, e = at % EIGHTS;
            float f[8];
            if (closed) {
                const uint8_t *src = page_smem + n * kCacheBlock * DH;
                if (n < 2) {
                    const uint32_t w[2] = {*reinterpret_cast<const uint32_t *>(src + cache_tile_byte(r, 8 * e, DH)), *reinterpret_cast<const uint32_t *>(src + cache_tile_byte(r, 8 * e + 4, DH))};
#pragma unroll
                    for (int b = 0; b < 8; ++b) f[b] = (float)(int8_t)(w[b >> 2] >> (8 * (b & 3))) * sc[n];
                } else {
#pragma unroll
                    for (int b = 0; b < 8; ++b) f[b] = (float)(int8_t)src[cache_tile_byte(8 * e + b, r, kCacheBlock)] * sc[n];
                }
            } else {
                unpack8(*reinterpret_cast<const uint4 *>(open + ((size_t)n * kCacheBlock + r) * DH + 8 * cache_open_eight(r, e)), f);
            }
            const size_t o = n < 2 ? (out0 + at / EIGHTS) * kw + ((size_t)n * H + head) * DH + 8 * e : (out0 + at / EIGHTS) * vw + (size_t)head * DH + 8 * e;
            void *base = n < 2 ? k_out : v_out;
            if (BF16) {
                uint32_t w[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * b], f[2 * b + 1]);
                    w[b] = *reinterpret_cast<const uint32_t *>(&p);
                }
                *reinterpret_cast<uint4 *>(reinterpret_cast<__nv_bfloat16 *>(base) + o) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                float4 *dst = reinterpret_cast<float4 *>(reinterpret_cast<float *>(base) + o);
                dst[0] = make_float4(f[0], f[1], f[2], f[3]);
                dst[1] = make_float4(f[4], f[5], f[6], f[7]);
            }
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
// met in full takes none.
constexpr int kReserveThreads = 1024, kReserveStep = 16;  // reference counts a thread looks at in one step

__global__ void __launch_bounds__(kReserveThreads) cache_reserve_kernel(CacheView c, const int32_t *__restrict__ slots, const int32_t *__restrict__ tokens, int n, int32_t *granted,
                                                                        unsigned int *status) {
    __shared__ int slot_of[kCacheMaxSeqs], upto[kCacheMaxSeqs], held_of[kCacheMaxSeqs], sums[32];
    __shared__ long long wide[32];
    __shared__ int dealt_smem;
    const int tid = threadIdx.x;
    const int slot = tid < n ? slots[tid] : -1;
    slot_of[tid] = slot;
    if (tid == 0) dealt_smem = 0;
    __syncthreads();
    bool able = tid < n && slot != -1;
    if (able && (slot < 0 || slot >= c.n_slots)) {
        atomicOr(status, kStatusCache);
        able = false;
    }
    for (int j = 0; j < tid && able; ++j) able = slot_of[j] != slot;
    int need = 0, held = 0;
    if (able) {
        held = c.held[slot];
        const int want = tokens[tid];
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
        long long before = 0, all = 0;
        for (int w = 0; w < 32; ++w) {
            if (w < warp) before += wide[w];
            all += wide[w];
        }
        upto[tid] = (int)min(s + before, 0x7fffffffll);
        held_of[tid] = held;
        total = (int)min(all, 0x7fffffffll);
    }
    __syncthreads();
    constexpr int STEP = kReserveThreads * kReserveStep;
    int found = 0;
    if (total > 0)
        for (long long p0 = 0; p0 < c.n_pages && found < total; p0 += STEP) {
            int mine = 0;
#pragma unroll
            for (int u = 0; u < kReserveStep; ++u) {
                const long long p = p0 + tid * kReserveStep + u;
                mine += p < c.n_pages && c.refs[p] == 0;
            }
            int sum;
            block_exclusive_sum(mine, sums, &sum);
            found += sum;
        }
    const bool met = able && (need == 0 || upto[tid] <= found);
    if (granted && tid < n) granted[tid] = met;
    // pages dealt: as far as the requests that are met reach
    if (met && need) atomicMax(&dealt_smem, upto[tid]);
    __syncthreads();
    const int dealt = dealt_smem;
    int base = 0;
    for (long long p0 = 0; p0 < c.n_pages && base < dealt; p0 += STEP) {
        uint32_t free_mask = 0;
#pragma unroll
        for (int u = 0; u < kReserveStep; ++u) {
            const long long p = p0 + tid * kReserveStep + u;
            if (p < c.n_pages && c.refs[p] == 0) free_mask |= 1u << u;
        }
        int sum, rank = base + block_exclusive_sum(__popc(free_mask), sums, &sum);
        base += sum;
        for (; free_mask && rank < dealt; free_mask &= free_mask - 1, ++rank) {
            const int p = (int)(p0 + tid * kReserveStep + __ffs(free_mask) - 1);
            int lo = 0, hi = n - 1;  // the first request whose running sum is above the rank
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (upto[mid] > rank) hi = mid; else lo = mid + 1;
            }
            const int before = lo ? upto[lo - 1] : 0;
            c.table[(size_t)slot_of[lo] * c.max_pages + held_of[lo] + rank - before] = p;
            c.refs[p] = 1;
        }
    }
    if (met && need) c.held[slot] = held + need;
}

__global__ void __launch_bounds__(256) cache_free_kernel(CacheView c, const int32_t *__restrict__ slots, unsigned int *status) {
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

// A block of threads copies the open rows of one K/V head; the first of a pair also shares the pages, and the last to have read the state changes it.
template <int DH>
__global__ void __launch_bounds__(256) cache_fork_kernel(CacheView c, const int32_t *__restrict__ srcs, const int32_t *__restrict__ dsts, int n, int32_t *done, unsigned int *status) {
    const int i = blockIdx.x, head = blockIdx.y, tid = threadIdx.x, H = c.H, src = srcs[i], dst = dsts[i];
    bool clash = false;
    for (int j = tid; j < n; j += blockDim.x) clash = clash || (j < i && dsts[j] == dst) || dsts[j] == src;
    clash = __syncthreads_or(clash);
    const bool skip = src == -1 || dst == -1, off = !skip && (src < 0 || src >= c.n_slots || dst < 0 || dst >= c.n_slots);
    int held = 0, length = 0;
    bool empty = false, sane = false;
    if (!skip && !off && !clash) {
        held = c.held[src];
        length = c.length[src];
        empty = c.held[dst] == 0 && c.length[dst] == 0;
        sane = cache_slot_ok(c, held, length);
    }
    const int full = length >> 6, rows = length & 63;
    bool bad_page = false;
    if (empty && sane) {
        for (int b = tid; b < full; b += blockDim.x) {
            const int page = c.table[(size_t)src * c.max_pages + b];
            bad_page = bad_page || page < 0 || page >= c.n_pages;
        }
    }
    bad_page = __syncthreads_or(bad_page);
    if (!empty || !sane || bad_page) {
        if (head == 0 && tid == 0) {
            if (done) done[i] = 0;
            if (off || (empty && !sane) || bad_page) atomicOr(status, kStatusCache);
        }
        return;
    }
    const uint4 *from = reinterpret_cast<const uint4 *>(c.open + ((size_t)src * H + head) * (3 * kCacheBlock * DH));
    uint4 *to = reinterpret_cast<uint4 *>(c.open + ((size_t)dst * H + head) * (3 * kCacheBlock * DH));
    const int per = rows * (DH / 8);
#pragma unroll 4
    for (int at = tid; at < 3 * per; at += blockDim.x) {
        const int t = at / per, j = t * kCacheBlock * (DH / 8) + at - t * per;
        to[j] = from[j];
    }
    if (head == 0)
        for (int b = tid; b < full; b += blockDim.x) {
            const int page = c.table[(size_t)src * c.max_pages + b];
            c.table[(size_t)dst * c.max_pages + b] = page;
            atomicAdd(c.refs + page, 1);
        }
    __syncthreads();
    if (tid == 0 && last_arrival(c.arrivals + dst, H)) {
        c.held[dst] = full;
        c.length[dst] = length;
        if (done) done[i] = 1;
    }
}

static hgf_status launched() { return cudaGetLastError() == cudaSuccess ? HGF_OK : HGF_ERR_CUDA; }

}  // namespace hgf

using namespace hgf;

extern "C" hgf_status hgf_cache_reserve(const hgf_cache *cache, const int32_t *slots, const int32_t *tokens, int64_t n, int32_t *granted, void *stream) {
    CacheView c;
    if (!slots || !tokens) return HGF_ERR_INVALID_ARG;
    if (const hgf_status st = parse_cache(cache, n, &c)) return st;
    unsigned int *status = device_status_word();
    if (!status) return HGF_ERR_CUDA;
    cache_reserve_kernel<<<1, kReserveThreads, 0, (cudaStream_t)stream>>>(c, slots, tokens, (int)n, granted, status);
    count_launch();
    return launched();
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
    const dim3 grid((unsigned)(n_rows / kCacheBlock + n_seqs), (unsigned)c.H);
    auto kernel = cache->head_dim == 64 ? cache_append_kernel<64> : cache_append_kernel<128>;
    kernel<<<grid, kAppendThreads, 0, (cudaStream_t)stream>>>(c, (const __nv_bfloat16 *)k, (const __nv_bfloat16 *)v, (int)n_rows, slots, starts, (int)n_seqs, done, status);
    count_launch();
    return launched();
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
    const dim3 grid((unsigned)(n_rows / kCacheBlock + 2 * n_seqs), (unsigned)c.H);
    const bool bf16 = (flags & HGF_FLAG_OUT_BF16) != 0;
    auto kernel = cache->head_dim == 64 ? (bf16 ? cache_read_kernel<64, true> : cache_read_kernel<64, false>) : (bf16 ? cache_read_kernel<128, true> : cache_read_kernel<128, false>);
    kernel<<<grid, kReadThreads, 0, (cudaStream_t)stream>>>(c, slots, first, starts, (int)n_seqs, (int)n_rows, k_out, v_out, status);
    count_launch();
    return launched();
}

extern "C" hgf_status hgf_cache_fork(const hgf_cache *cache, const int32_t *src, const int32_t *dst, int64_t n, int32_t *done, void *stream) {
    CacheView c;
    if (!src || !dst) return HGF_ERR_INVALID_ARG;
    if (const hgf_status st = parse_cache(cache, n, &c)) return st;
    unsigned int *status = device_status_word();
    if (!status) return HGF_ERR_CUDA;
    auto kernel = cache->head_dim == 64 ? cache_fork_kernel<64> : cache_fork_kernel<128>;
    kernel<<<dim3((unsigned)n, (unsigned)c.H), 256, 0, (cudaStream_t)stream>>>(c, src, dst, (int)n, done, status);
    count_launch();
    return launched();
}

extern "C" hgf_status hgf_cache_free(const hgf_cache *cache, const int32_t *slots, int64_t n, void *stream) {
    CacheView c;
    if (!slots) return HGF_ERR_INVALID_ARG;
    if (const hgf_status st = parse_cache(cache, n, &c)) return st;
    unsigned int *status = device_status_word();
    if (!status) return HGF_ERR_CUDA;
    cache_free_kernel<<<(unsigned)n, 256, 0, (cudaStream_t)stream>>>(c, slots, status);
    count_launch();
    return launched();
}
