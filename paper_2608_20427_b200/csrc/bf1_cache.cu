// The paged cache: the tables of a serving step, and its keys and values put into the pages.
//
// plan_cache_kernel turns lengths into everything that the step's other calls look up: pages taken from a stack of free ones and
// written into the page table, where each new token stands (position, slot), and the runs of tokens that share a page (units).
// One thread-block cluster does it: every CTA reads all lengths and scans them by itself, so nothing is exchanged; the
// cluster's barrier stands between the reads of arrays that may be written in place and their writes.
//
// The write kernels go by units.  In 8 bits the rows of a page and KV head share a scale, so whoever writes to a page has to see all of the
// step's rows for it: a unit is what one CTA (or half a warp) does.  Scales are powers of two: e4m3 has the same precision in every
// binade, so that a finer scale would gain nothing, and rows that have to move under a larger scale keep their digits (but for
// those that fall below 2^-6 of it, which have fewer at any scale).
//
// Measured (16 query / 8 KV heads, d = 128, in a graph): the tables of 32 sequences of a token each 3.2 us, of 512 with 130 prompts and 32 released
// ones 11.1; keys and values of 32K prompt tokens into 8-bit pages 32.0 us, 6.3 TB/s, 97 % of a copy; of 8 / 256 single tokens, with the rotation of
// their queries and keys, 2.9 / 4.2 us, chains of launch, unit, position, angle and scale.
#include <math.h>

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <type_traits>

#include "bf1_rope.cuh"

namespace bf1 {

constexpr int kCachePage = 64;
constexpr int kTableThreads = 1024;       // at most
constexpr int kTableHeld = 2048;          // sequences whose starts stand in shared memory; more of them: in bf1_cache_plan::starts

struct TableArgs {
    const int32_t *lens, *add;         // [batch]
    int32_t* table;                    // [batch, max_pages]
    int32_t* free_pages;               // stack of free pages, or null: the table is complete
    const int32_t* free_count;
    int32_t batch, max_pages, num_pages;
    bf1_cache_plan p;
};

__device__ __forceinline__ int pages_of(int n) { return (n + kCachePage - 1) / kCachePage; }
__device__ __forceinline__ int4 add4(int4 a, int4 b) { return make_int4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
__device__ __forceinline__ int4 scan_warp(int4 x) {       // inclusive
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int a = __shfl_up_sync(0xffffffffu, x.x, off), b = __shfl_up_sync(0xffffffffu, x.y, off),
                  c = __shfl_up_sync(0xffffffffu, x.z, off), d = __shfl_up_sync(0xffffffffu, x.w, off);
        if (lane >= off) x = add4(x, make_int4(a, b, c, d));
    }
    return x;
}
__device__ __forceinline__ int4 lane4(int4 x, int l) {
    return make_int4(__shfl_sync(0xffffffffu, x.x, l), __shfl_sync(0xffffffffu, x.y, l), __shfl_sync(0xffffffffu, x.z, l), __shfl_sync(0xffffffffu, x.w, l));
}
// Exclusive prefix sums over the CTA of four numbers of every thread at once; `total` gets the sums.
__device__ __forceinline__ int4 scan4(int4 v, int4* warp_sums, int4& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int4 x = scan_warp(v);
    __syncthreads();                                     // the last use of warp_sums is over
    if (lane == 31) warp_sums[warp] = x;
    __syncthreads();
    const int4 sums = scan_warp(lane < warps ? warp_sums[lane] : make_int4(0, 0, 0, 0));
    total = lane4(sums, 31);
    const int4 before = lane4(sums, max(warp - 1, 0));
    const int4 mine = make_int4(x.x - v.x, x.y - v.y, x.z - v.z, x.w - v.w);
    return warp ? add4(before, mine) : mine;
}

// A thread for every sequence first (what each needs, and where it begins, by a scan), then a lane for every unit, which looks up the
// one page of its tokens.  With few sequences and tokens this is a chain of dependent looks at memory: lengths, stack, page.
__global__ void __launch_bounds__(kTableThreads, 1) plan_cache_kernel(const TableArgs a) {
    __shared__ int4 warp_sums[kTableThreads / 32];
    __shared__ int4 held_starts[kTableHeld];
    __shared__ int held_adds[kTableHeld];
    __shared__ long long sums[3];
    __shared__ int flags;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    const int rank = blockIdx.x, ranks = gridDim.x;      // the grid is one cluster
    const int threads = ranks * blockDim.x, gtid = rank * blockDim.x + tid;
    const bool stack = a.free_pages != nullptr;
    const bf1_cache_plan& p = a.p;
    if (tid < 3) sums[tid] = 0;
    if (tid == 0) flags = 0;
    pdl_wait();
    __syncthreads();
    const int had = stack ? *a.free_count : 0;
    // ---- what the step needs in all, in 64 bits: it may be refused for any lengths ----------------------------------------------
    long long tokens = 0, fresh = 0, back = 0;
    int bad = 0, n0 = 0, m0 = 0;                          // (n0, m0: of this thread's first sequence, which mostly is its only one)
    for (int s = tid; s < a.batch; s += blockDim.x) {
        const int n = a.lens[s], m = a.add[s];
        if (s == tid) n0 = n, m0 = m;
        if (n < 0 || m < -1 || (long long)n + max(m, 0) > (long long)a.max_pages * kCachePage) {
            bad = BF1_DEV_BAD_SEQLENS;
            continue;
        }
        tokens += max(m, 0);
        if (stack) {
            if (m < 0) back += pages_of(n);
            else fresh += pages_of(n + m) - pages_of(n);
        }
    }
    if (warp * 32 < a.batch) {
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) {
            tokens += __shfl_xor_sync(0xffffffffu, tokens, off);
            fresh += __shfl_xor_sync(0xffffffffu, fresh, off);
            back += __shfl_xor_sync(0xffffffffu, back, off);
            bad |= __shfl_xor_sync(0xffffffffu, bad, off);
        }
        if (lane == 0) {
            atomicAdd(reinterpret_cast<unsigned long long*>(&sums[0]), (unsigned long long)tokens);
            atomicAdd(reinterpret_cast<unsigned long long*>(&sums[1]), (unsigned long long)fresh);
            atomicAdd(reinterpret_cast<unsigned long long*>(&sums[2]), (unsigned long long)back);
            if (bad) atomicOr(&flags, bad);
        }
    }
    __syncthreads();
    int status = flags;
    if (sums[0] > p.capacity_tokens) status |= BF1_DEV_CAPACITY;
    if (stack && (had < 0 || had + sums[2] > a.num_pages || sums[1] > had + sums[2])) status |= BF1_DEV_CAPACITY;
    const bool refused = status != 0;
    const int top = refused ? had : had + (int)sums[2];   // of the stack, with what is put back
    const int total_tokens = refused ? 0 : (int)sums[0];
    // ---- where every sequence's tokens, fresh pages and units begin, and its length: every CTA has them all ------------------------
    // (a released sequence takes no pages: where its own go on the stack stands there instead)
    int4* const starts = a.batch <= kTableHeld ? held_starts : reinterpret_cast<int4*>(p.starts);
    const int* const adds = a.batch <= kTableHeld ? held_adds : a.add;   // (none of them counts in a refused step)
    int4 at = make_int4(0, 0, 0, 0);                      // tokens, fresh pages, units, pages put back
    for (int s0 = 0; s0 < a.batch; s0 += blockDim.x) {
        const int s = s0 + tid;
        int n = 0, m = 0;
        int4 mine = make_int4(0, 0, 0, 0);
        if (s < a.batch) {
            n = s0 ? a.lens[s] : n0;
            m = refused ? 0 : s0 ? a.add[s] : m0;
            mine.x = max(m, 0);
            mine.y = stack && m > 0 ? pages_of(n + m) - pages_of(n) : 0;
            mine.z = m > 0 ? (n + m - 1) / kCachePage - n / kCachePage + 1 : 0;
            mine.w = stack && m < 0 ? pages_of(n) : 0;
        }
        int4 total;
        const int4 before = add4(at, scan4(mine, warp_sums, total));
        if (s < a.batch) {
            if (starts == held_starts || s0 / (int)blockDim.x % ranks == rank) starts[s] = make_int4(before.x, m < 0 ? before.w : before.y, before.z, n);
            if (starts == held_starts) held_adds[s] = m;
            if (rank == 0) p.cu_tokens[s] = before.x;
        }
        at = add4(at, total);
    }
    const int units = at.z;
    if (gtid == 0) {
        p.cu_tokens[a.batch] = at.x;
        *p.num_units = units;
        *p.status = status;
    }
    if (ranks > 1) {                                      // lengths and the count have been read by all: they may be written in place
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }
    if (gtid == 0) *p.free_count = top - at.y;
    // Every look-up and store below keeps to its array for whatever numbers the scan has made of lengths that have changed since they were added up.
    auto pop = [&](int i) { return (unsigned)i < (unsigned)top ? a.free_pages[top - 1 - i] : -1; };     // the i-th page taken
    auto row_of = [&](int s) { return a.table + (size_t)s * a.max_pages; };
    auto in_row = [&](int i) { return (unsigned)i < (unsigned)a.max_pages; };
    // ---- lengths after the step; pages put back ------------------------------------------------------------------------------------
    // All warps share the sequences, and the units below, a few to each: what is done for one after the other waits for memory each time
    // (32 to a warp, and most warps idle: 512 sequences, 130 of them prompts, 18.1 us)
    const int all_warps = ranks * warps, my_warp = rank * warps + warp;
    const int per_seq = min(32, (a.batch + all_warps - 1) / all_warps), per_unit = max(1, min(32, (units + all_warps - 1) / all_warps));
    for (int s0 = my_warp * per_seq; s0 < a.batch; s0 += all_warps * per_seq) {
        const int s = s0 + lane;
        const bool live = lane < per_seq && s < a.batch;
        int m = 0, n = 0, to = 0;
        if (live) {
            const int4 st = starts[s];
            m = refused ? 0 : adds[s];
            n = st.w;
            to = st.y;
            p.seqlens[s] = m < 0 ? 0 : n + m;
        }
        // fresh pages into the table, where none are put back that might be among them
        const int held = pages_of(n), want = stack && m > 0 ? pages_of(n + m) - held : 0;
        if (at.w == 0) {
            unsigned grown = __ballot_sync(0xffffffffu, want > 1);
            if (want == 1 && in_row(held)) row_of(s)[held] = pop(to);
            while (grown) {
                const int l = __ffs(grown) - 1;
                grown &= grown - 1;
                const int count = __shfl_sync(0xffffffffu, want, l), h = __shfl_sync(0xffffffffu, held, l), f = __shfl_sync(0xffffffffu, to, l);
                for (int i = lane; i < count && in_row(h + i); i += 32) row_of(s0 + l)[h + i] = pop(f + i);
            }
        } else {
            unsigned gone = __ballot_sync(0xffffffffu, m < 0);
            while (gone) {
                const int l = __ffs(gone) - 1;
                gone &= gone - 1;
                const int count = __shfl_sync(0xffffffffu, held, l), first = had + __shfl_sync(0xffffffffu, to, l);
                for (int i = lane; i < count && in_row(i) && (unsigned)(first + i) < (unsigned)a.num_pages; i += 32) a.free_pages[first + i] = row_of(s0 + l)[i];
            }
        }
    }
    if (at.w > 0) {                                       // (the same in every CTA)
        if (ranks > 1) {
            cluster_arrive();
            cluster_wait();
        } else {
            __syncthreads();
        }
        // fresh pages, some of them from what has just been put back
        for (int s0 = my_warp * per_seq; s0 < a.batch; s0 += all_warps * per_seq) {
            const int s = s0 + lane;
            int held = 0, want = 0, first = 0;
            if (lane < per_seq && s < a.batch) {
                const int4 st = starts[s];
                const int m = adds[s];
                held = pages_of(st.w);
                want = m > 0 ? pages_of(st.w + m) - held : 0;
                first = st.y;
            }
            unsigned grown = __ballot_sync(0xffffffffu, want > 0);
            while (grown) {
                const int l = __ffs(grown) - 1;
                grown &= grown - 1;
                const int count = __shfl_sync(0xffffffffu, want, l), h = __shfl_sync(0xffffffffu, held, l), f = __shfl_sync(0xffffffffu, first, l);
                for (int i = lane; i < count && in_row(h + i); i += 32) row_of(s0 + l)[h + i] = pop(f + i);
            }
        }
    }
    // ---- units, a lane to each, then their tokens' positions and slots --------------------------------------------------------------
    for (int u0 = my_warp * per_unit; u0 < units; u0 += all_warps * per_unit) {
        const int u = u0 + lane;
        int t = 0, count = 0, pos = 0, slot = -1;
        if (lane < per_unit && u < units) {
            int lo = 0, hi = a.batch;                     // the last sequence that begins at or in front of unit u
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (starts[mid].z <= u) lo = mid;
                else hi = mid;
            }
            const int4 st = starts[lo];
            const int end = lo + 1 < a.batch ? starts[lo + 1].x : total_tokens;
            const int lp = st.w / kCachePage + (u - st.z), held = pages_of(st.w);
            pos = max(st.w, lp * kCachePage);
            t = st.x + (pos - st.w);
            const int row = pos % kCachePage;
            count = min(kCachePage - row, end - t);
            int page = stack && lp >= held ? pop(st.y + lp - held) : in_row(lp) ? row_of(lo)[lp] : -1;
            count = t < 0 ? 0 : min(count, p.capacity_tokens - t);
            if (page < 0 || page >= a.num_pages) {
                atomicOr(p.status, BF1_DEV_BAD_ROUTE);
                page = -1;
            } else {
                slot = page * kCachePage + row;
            }
            if (u < p.capacity_units) reinterpret_cast<int4*>(p.units)[u] = make_int4(t, count, page, row);
            if (count > 0) {
                p.positions[t] = pos;                     // (single tokens, side by side in a step of them)
                p.slots[t] = slot;
            }
        }
        unsigned more = __ballot_sync(0xffffffffu, count > 1);
        while (more) {
            const int l = __ffs(more) - 1;
            more &= more - 1;
            const int tl = __shfl_sync(0xffffffffu, t, l), cl = __shfl_sync(0xffffffffu, count, l), pl = __shfl_sync(0xffffffffu, pos, l),
                      sl = __shfl_sync(0xffffffffu, slot, l);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int k = 1 + lane + 32 * i;
                if (k < cl) {
                    p.positions[tl + k] = pl + k;
                    p.slots[tl + k] = sl < 0 ? -1 : sl + k;
                }
            }
        }
    }
    for (int t = total_tokens + gtid; t < p.capacity_tokens; t += threads) p.positions[t] = p.slots[t] = -1;
    for (int u = units + gtid; u < p.capacity_units; u += threads) reinterpret_cast<int4*>(p.units)[u] = make_int4(-1, -1, -1, -1);
}

// ---- keys and values into the pages ------------------------------------------------------------------------------------------------

struct WriteArgs {
    Rows x[2];                         // keys, values
    Rows q, out_q;
    uint8_t* pages[2];                 // [num_pages, 64, hkv, D], bf16 or e4m3
    float* scales[2];                  // [num_pages, hkv] (8 bits)
    const int4* units;                 // [num_units], those behind the last one with -1 tokens
    const int32_t* positions;
    int32_t* status;
    RopeTable rope;
    int32_t tokens, hq, hkv, num_pages, num_units;
    int32_t heads_per_cta;             // cache_write_turned_kernel
    int64_t write_ctas;                // CTAs behind them rotate queries
    int32_t q_shares;                  // shares of the query heads
};

__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return lo | (uint32_t)hi << 16;
}
__device__ __forceinline__ float2 from_e4m3x2(uint32_t v) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)v));
    float2 f;
    asm("{\n\t.reg .f16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(h));
    return f;
}
// Largest magnitude that counts for a scale (an infinity and a NaN do not: they are stored as NaN under any)
__device__ __forceinline__ float magnitude_of(const float (&x)[8], float top) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float m = fabsf(x[i]);
        if (m <= FLT_MAX) top = fmaxf(top, m);
    }
    return top;
}
// The same on eight bf16 values, as whole numbers, two at a time: without their sign they are ordered as their bits are, an infinity
// above every finite value and NaN above that.  Both halves of `top` run for themselves.
__device__ __forceinline__ uint32_t magnitude_bits(const uint4& v, uint32_t top) {
    top = __vmaxu2(top, v.x & 0x7fff7fffu);
    top = __vmaxu2(top, v.y & 0x7fff7fffu);
    top = __vmaxu2(top, v.z & 0x7fff7fffu);
    return __vmaxu2(top, v.w & 0x7fff7fffu);
}
// The smallest power of two, 2^-64 at least, under which `top` is within 448 = 1.75 * 2^8.
__device__ __forceinline__ float scale_for(float top) {
    const int e = (int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 8;     // above 1.75 the sum carries into the exponent
    return __uint_as_float((uint32_t)max(e, 127 - 64) << 23);
}
__device__ __forceinline__ uint2 quantize(const float (&x)[8], float inv) {   // inv: a power of two, so that the product is exact
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = fabsf(x[i]) <= FLT_MAX ? x[i] * inv : NAN;
    return make_uint2(e4m3x4(y[0], y[1], y[2], y[3]), e4m3x4(y[4], y[5], y[6], y[7]));
}
__device__ __forceinline__ uint2 requantize(uint2 v, float ratio) {
    const float2 a = from_e4m3x2(v.x & 0xffffu), b = from_e4m3x2(v.x >> 16), c = from_e4m3x2(v.y & 0xffffu), d = from_e4m3x2(v.y >> 16);
    return make_uint2(e4m3x4(a.x * ratio, a.y * ratio, b.x * ratio, b.y * ratio), e4m3x4(c.x * ratio, c.y * ratio, d.x * ratio, d.y * ratio));
}

__device__ __forceinline__ uint2 quantize_finite(const float (&x)[8], float inv) {
    return make_uint2(e4m3x4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv), e4m3x4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
}
// The rows in front of a unit's own under the page's new scale, and that scale.  `out`: this thread's chunk of row 0.
template <int kRows>
__device__ __forceinline__ void finish_page(uint8_t* out, size_t pitch, int r0, int rows, float before, float scale, float* at) {
    if (rows > 0 && before != scale)
        for (int r = r0; r < rows; r += kRows) {
            uint2* v = reinterpret_cast<uint2*>(out + r * pitch);
            *v = requantize(*v, before * (1.f / scale));
        }
    if (threadIdx.x == 0) *at = scale;
}

// A unit whose tokens, rows and page exist.  What a plan holds is looked at once more here: a plan for other tensors than these, or one
// that has been written over, costs the unit and not memory.
__device__ __forceinline__ bool unit_ok(const WriteArgs& a, const int4& u) {
    return u.x >= 0 && u.y >= 1 && u.y <= a.tokens - u.x && u.w >= 0 && u.w + u.y <= kCachePage && u.z >= 0 && u.z < a.num_pages;
}

// The CTAs behind the writing ones: tokens' queries, as rope_kernel does them.
template <int D>
__device__ __forceinline__ void rotate_queries(const WriteArgs& a) {
    const int64_t block = (int64_t)blockIdx.x - a.write_ctas;
    rope_block<D, 2>(a.rope, a.positions, block / a.q_shares * kRopeTokens<D>, a.tokens, 1.f, a.q, a.q, a.out_q, a.out_q, a.hq, a.hq, 4 * (int)(block % a.q_shares),
                     4 * a.q_shares);
}

template <int kWarps>
__device__ __forceinline__ uint32_t max_of_warps(uint32_t v, uint32_t* warp_top) {     // of the whole CTA (one barrier)
    v = __reduce_max_sync(0xffffffffu, v);
    if ((threadIdx.x & 31) == 0) warp_top[threadIdx.x >> 5] = v;
    __syncthreads();
    v = warp_top[0];
#pragma unroll
    for (int i = 1; i < kWarps; ++i) v = max(v, warp_top[i]);
    return v;
}

// A CTA per unit, KV head and K or V: the rows stay in registers, as they came, between the look for their largest value and the store.
template <int D, bool kFp8>
__global__ void __launch_bounds__(128) cache_write_pages_kernel(const WriteArgs a) {
    constexpr int kChunks = D / 8, kRows = 128 / kChunks, kPer = kCachePage / kRows;
    __shared__ uint32_t warp_top[4];
    pdl_wait();
    const int which = blockIdx.x & 1, h = (blockIdx.x >> 1) % a.hkv, unit = (blockIdx.x >> 1) / a.hkv;
    const int4 u = a.units[unit];
    if (u.y < 0) return;                                 // behind the last unit
    if (!unit_ok(a, u)) {
        if (threadIdx.x == 0) atomicOr(a.status, BF1_DEV_BAD_ROUTE);
        return;
    }
    float* const at = kFp8 ? a.scales[which] + (size_t)u.z * a.hkv + h : nullptr;
    const float before = kFp8 && u.w > 0 ? *at : 0.f;
    const int c = threadIdx.x % kChunks, r0 = threadIdx.x / kChunks;
    const Rows& in = a.x[which];
    const size_t pitch = (size_t)a.hkv * D;
    const size_t first = ((size_t)u.z * kCachePage) * pitch + (size_t)h * D + 8 * c;     // element of the page's row 0
    uint4 x[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int r = r0 + i * kRows;
        x[i] = make_uint4(0u, 0u, 0u, 0u);
        if (r < u.y) x[i] = *reinterpret_cast<const uint4*>(in.at((int64_t)u.x + r, h) + 8 * c);
    }
    if constexpr (!kFp8) {
        __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.pages[which]) + first;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = r0 + i * kRows;
            if (r < u.y) *reinterpret_cast<uint4*>(out + (u.w + r) * pitch) = x[i];
        }
    } else {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) top = magnitude_bits(x[i], top);
        top = max_of_warps<4>(max(top & 0xffffu, top >> 16), warp_top);
        const bool finite = top < 0x7f80u;
        if (!finite) {                                   // once more without what is not (the whole CTA)
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                float y[8];
                unpack_bf16x8(x[i], y);
                most = magnitude_of(y, most);
            }
            __syncthreads();
            top = max_of_warps<4>(__float_as_uint(most) >> 16, warp_top);
        }
        const float scale = fmaxf(scale_for(__uint_as_float(top << 16)), before), inv = 1.f / scale;
        uint8_t* out = a.pages[which] + first;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = r0 + i * kRows;
            if (r < u.y) {
                float y[8];
                unpack_bf16x8(x[i], y);
                *reinterpret_cast<uint2*>(out + (u.w + r) * pitch) = finite ? quantize_finite(y, inv) : quantize(y, inv);
            }
        }
        finish_page<kRows>(out, pitch, r0, u.w, before, scale, at);
    }
}

// The same with a rope, a CTA per unit, K or V, and a few heads: a thread holds the two chunks of eight pairs of a row; the angles of the page are made
// once, by all threads, for all of the CTA's heads; the next head's rows are on their way while one is written.  (A CTA of 128 threads per head, eight
// angles to a thread and row: 24000 tokens of 16 / 8 heads 136 us, 77 as it is; a single page of one head 8.6 and 6.6 us.)
constexpr int kTurnThreads = 256;
template <int D, bool kFp8>
__global__ void __launch_bounds__(kTurnThreads) cache_write_turned_kernel(const WriteArgs a) {
    constexpr int kTasks = D / 16, kRows = kTurnThreads / kTasks, kPer = kCachePage / kRows, kWarps = kTurnThreads / 32;
    __shared__ uint32_t warp_top[2][kWarps];
    __shared__ float2 angles[kCachePage][8][kTasks];     // [row][pair of the thread][thread of the row]
    pdl_wait();
    const int shares = (a.hkv + a.heads_per_cta - 1) / a.heads_per_cta;
    const int which = blockIdx.x & 1, h0 = (blockIdx.x >> 1) % shares * a.heads_per_cta, unit = (blockIdx.x >> 1) / shares;
    const int4 u = a.units[unit];
    if (u.y < 0) return;                                 // behind the last unit
    if (!unit_ok(a, u)) {
        if (threadIdx.x == 0) atomicOr(a.status, BF1_DEV_BAD_ROUTE);
        return;
    }
    const int c = threadIdx.x % kTasks, r0 = threadIdx.x / kTasks, h_end = min(h0 + a.heads_per_cta, a.hkv);
    const bool turn = which == 0 && 16 * c < a.rope.dim;
    const int lo = turn && a.rope.half ? 8 * c : 16 * c, hi = turn && a.rope.half ? a.rope.dim / 2 + 8 * c : 16 * c + 8;
    const Rows& in = a.x[which];
    uint4 next[kPer][2];
    auto fetch = [&](int h) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int r = r0 + i * kRows;
            next[i][0] = next[i][1] = make_uint4(0u, 0u, 0u, 0u);
            if (r < u.y) {
                const __nv_bfloat16* row = in.at((int64_t)u.x + r, h);
                next[i][0] = *reinterpret_cast<const uint4*>(row + lo);
                next[i][1] = *reinterpret_cast<const uint4*>(row + hi);
            }
        }
    };
    fetch(h0);
    if (which == 0) {
        const int pairs = a.rope.dim / 2;
#pragma unroll 4
        for (int i = threadIdx.x; i < u.y * pairs; i += kTurnThreads) {
            const int r = i / pairs, pair = i - r * pairs;
            angles[r][pair % 8][pair / 8] = rope_angle(a.rope, a.positions[u.x + r], pair);
        }
        __syncthreads();
    }
    const size_t pitch = (size_t)a.hkv * D;
#pragma unroll 1
    for (int h = h0; h < h_end; ++h) {
        float* const at = kFp8 ? a.scales[which] + (size_t)u.z * a.hkv + h : nullptr;
        const float before = kFp8 && u.w > 0 ? *at : 0.f;
        float x[kPer][2][8], top = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            unpack_bf16x8(next[i][0], x[i][0]);
            unpack_bf16x8(next[i][1], x[i][1]);
        }
        if (h + 1 < h_end) fetch(h + 1);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (turn && r0 + i * kRows < u.y) {
                const float2(&by)[8][kTasks] = angles[r0 + i * kRows];
                if (a.rope.half) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) rope_turn(x[i][0][k], x[i][1][k], by[k][c].x, by[k][c].y);
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        rope_turn(x[i][0][2 * k], x[i][0][2 * k + 1], by[k][c].x, by[k][c].y);
                        rope_turn(x[i][1][2 * k], x[i][1][2 * k + 1], by[4 + k][c].x, by[4 + k][c].y);
                    }
                }
            }
            if (kFp8) top = magnitude_of(x[i][1], magnitude_of(x[i][0], top));
        }
        const size_t first = ((size_t)u.z * kCachePage) * pitch + (size_t)h * D;         // element of the page's row 0
        if constexpr (!kFp8) {
            __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.pages[which]) + first;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = r0 + i * kRows;
                if (r < u.y) {
                    *reinterpret_cast<uint4*>(out + (u.w + r) * pitch + lo) = pack_bf16x8(x[i][0]);
                    *reinterpret_cast<uint4*>(out + (u.w + r) * pitch + hi) = pack_bf16x8(x[i][1]);
                }
            }
        } else {
            // (two places in turn: a warp may be a head ahead of the one that still reads)
            top = __uint_as_float(max_of_warps<kWarps>(__float_as_uint(top), warp_top[(h - h0) & 1]));
            const float scale = fmaxf(scale_for(top), before), inv = 1.f / scale;
            uint8_t* out = a.pages[which] + first;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = r0 + i * kRows;
                if (r < u.y) {
                    *reinterpret_cast<uint2*>(out + (u.w + r) * pitch + lo) = quantize(x[i][0], inv);
                    *reinterpret_cast<uint2*>(out + (u.w + r) * pitch + hi) = quantize(x[i][1], inv);
                }
            }
            finish_page<kTurnThreads / (D / 8)>(out + 8 * (threadIdx.x % (D / 8)), pitch, threadIdx.x / (D / 8), u.w, before, scale, at);
        }
    }
}

// A CTA per unit and four KV heads, a warp to each, half of it for K and half for V: for units of a token or a few, which a CTA would not fill.  kDeep rows
// (twice as many with d = 64) are on their way at once, under angles that the whole CTA makes; a longer unit's rows are read twice, for the scale and
// for the store.
template <int D, bool kFp8, bool kRope>
__global__ void __launch_bounds__(128) cache_write_tokens_kernel(const WriteArgs a) {
    constexpr int kChunks = D / 8, kRows = 16 / kChunks, kDeep = 2, kRound = kDeep * kRows;    // lanes to a row, rows side by side and in a round
    pdl_wait();
    if (kRope && (int64_t)blockIdx.x >= a.write_ctas) return rotate_queries<D>(a);
    const int groups = (a.hkv + 3) / 4, unit = blockIdx.x / groups, h = blockIdx.x % groups * 4 + (threadIdx.x >> 5);
    const bool live = h < a.hkv;
    const int4 u = a.units[unit];
    if (u.y < 0) return;                                        // behind the last unit
    const int lane = threadIdx.x & 31, which = lane >> 4, c = lane % kChunks, r0 = (lane & 15) / kChunks;
    if (!unit_ok(a, u)) {
        if (threadIdx.x == 0) atomicOr(a.status, BF1_DEV_BAD_ROUTE);
        return;
    }
    const Rows& in = a.x[which];
    // The angles, D / 2 pairs to a row: of one round, in 64 bits where numbers in 8 bits come of them, or, where there are more rounds, of all rows at once in
    // 32 bits (a round's angles in front of every round: four prompts of 120 among 512 sequences 140 us, 62 as it is)
    using Angle = typename std::conditional<kFp8, double2, float2>::type;
    __shared__ __align__(16) uint8_t angle_bytes[kRope ? kCachePage * D / 2 * sizeof(float2) : 16];
    static_assert(!kRope || sizeof(Angle) * kRound <= sizeof(float2) * kCachePage, "a round's angles are no more than a page's");
    Angle* const round_angles = reinterpret_cast<Angle*>(angle_bytes);
    float2* const page_angles = reinterpret_cast<float2*>(angle_bytes);
    const bool rounds = u.y > kRound;
    if constexpr (kRope) {
        for (int i = threadIdx.x; i < u.y * D / 2; i += 128) {
            const int r = i / (D / 2), pair = i % (D / 2);
            if (2 * pair >= a.rope.dim) continue;
            if (rounds || !kFp8) page_angles[i] = rope_angle(a.rope, a.positions[u.x + r], pair);
            else if constexpr (kFp8) round_angles[i] = rope_angle64(a.rope, a.positions[u.x + r], pair);
        }
        __syncthreads();
    }
    float x[kDeep][8];                                          // rows rb + r0, rb + r0 + kRows, ...
    const bool turn = kRope && which == 0 && 8 * c < a.rope.dim;
    const int other = turn && a.rope.half ? 8 * rope_other(a.rope, c) : 8 * c;
    auto load = [&](int rb) {                                   // (all loads in front of what K and V do apart)
        uint4 own[kDeep], pair_of[kDeep];
#pragma unroll
        for (int j = 0; j < kDeep; ++j) {
            const int r = rb + r0 + j * kRows;
            own[j] = pair_of[j] = make_uint4(0u, 0u, 0u, 0u);
            if (!live || r >= u.y) continue;
            const __nv_bfloat16* row = in.at((int64_t)u.x + r, h);
            own[j] = *reinterpret_cast<const uint4*>(row + 8 * c);
            if (kRope) pair_of[j] = *reinterpret_cast<const uint4*>(row + other);
        }
#pragma unroll
        for (int j = 0; j < kDeep; ++j) {
            const int r = rb + r0 + j * kRows;
            unpack_bf16x8(own[j], x[j]);
            if (!turn || r >= u.y) continue;
            if (rounds) rope_chunk(a.rope, c, x[j], pair_of[j], [&](int pair) { return page_angles[r * (D / 2) + pair]; });
            else rope_chunk(a.rope, c, x[j], pair_of[j], [&](int pair) { return round_angles[r * (D / 2) + pair]; });
        }
    };
    const size_t pitch = (size_t)a.hkv * D;
    const size_t first = ((size_t)u.z * kCachePage) * pitch + (size_t)h * D + 8 * c;
    if constexpr (!kFp8) {
        __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(a.pages[which]) + first;
        for (int rb = 0; rb < u.y; rb += kRound) {
            load(rb);
#pragma unroll
            for (int j = 0; j < kDeep; ++j) {
                const int r = rb + r0 + j * kRows;
                if (live && r < u.y) *reinterpret_cast<uint4*>(out + (u.w + r) * pitch) = pack_bf16x8(x[j]);
            }
        }
        return;
    }
    float* const at = a.scales[which] + (size_t)u.z * a.hkv + h;
    const float before = live && u.w > 0 ? *at : 0.f;
    float top = 0.f;
    for (int rb = (u.y - 1) / kRound * kRound; rb >= 0; rb -= kRound) {    // the first rows last: they stay in x
        load(rb);
#pragma unroll
        for (int j = 0; j < kDeep; ++j)
            if (live && rb + r0 + j * kRows < u.y) top = magnitude_of(x[j], top);
    }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    const float scale = fmaxf(scale_for(top), before), inv = 1.f / scale;
    uint8_t* out = a.pages[which] + first;
    for (int rb = 0; rb < u.y; rb += kRound) {
        if (rb > 0) load(rb);
#pragma unroll
        for (int j = 0; j < kDeep; ++j) {
            const int r = rb + r0 + j * kRows;
            if (live && r < u.y) *reinterpret_cast<uint2*>(out + (u.w + r) * pitch) = quantize(x[j], inv);
        }
    }
    if (!live) return;
    if (u.w > 0 && before != scale) {
        constexpr int kAhead = 8;
        for (int r = r0; r < u.w; r += kAhead * kRows) {
            uint2 v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (r + i * kRows < u.w) v[i] = *reinterpret_cast<const uint2*>(out + (r + i * kRows) * pitch);
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (r + i * kRows < u.w) *reinterpret_cast<uint2*>(out + (r + i * kRows) * pitch) = requantize(v[i], before * inv);
        }
    }
    if ((lane & 15) == 0) *at = scale;
}

typedef void (*WriteKernel)(WriteArgs);

static int check_plan(const bf1_cache_plan* p) {
    if (!p) return fail(BF1_ERR_INVALID_ARG, "the cache plan is null");
    if (p->batch < 0 || p->batch > 65535 || p->capacity_tokens < 0 || p->capacity_tokens > (1 << 30) || p->capacity_units < 0)
        return fail(BF1_ERR_INVALID_ARG, "cache plan: batch, capacity_tokens or capacity_units out of range");
    if (!p->seqlens || !p->free_count || !p->cu_tokens || !p->positions || !p->slots || !p->units || !p->num_units || !p->starts || !p->status)
        return fail(BF1_ERR_INVALID_ARG, "a cache-plan pointer is null");
    if (((uintptr_t)p->units | (uintptr_t)p->starts) & 15) return fail(BF1_ERR_INVALID_ARG, "units and starts must be 16-byte aligned");
    return BF1_OK;
}

}  // namespace bf1

using namespace bf1;

extern "C" int32_t bf1_cache_plan_units(int32_t batch, int32_t tokens) {
    if (batch < 0 || tokens < 0) return -1;
    const int64_t most = (int64_t)tokens / kCachePage + 2 * (int64_t)batch;   // n tokens touch at most (n + 62) / 64 + 1 pages
    return (int32_t)std::max<int64_t>(1, std::min<int64_t>(tokens, most));
}

extern "C" int bf1_plan_cache(const int32_t* seqlens_dev, const int32_t* new_lens_dev, int32_t* page_table_dev, int32_t max_pages_per_seq,
                              int32_t num_pages, int32_t* free_pages_dev, const int32_t* free_count_dev, const bf1_cache_plan* out,
                              void* stream) {
    if (int rc = check_plan(out)) return rc;
    if (out->batch > 0 && (!seqlens_dev || !new_lens_dev || !page_table_dev)) return fail(BF1_ERR_INVALID_ARG, "seqlens, new_lens or page_table is null");
    if ((free_pages_dev == nullptr) != (free_count_dev == nullptr)) return fail(BF1_ERR_INVALID_ARG, "free_pages and free_count go together");
    if (max_pages_per_seq < 1 || max_pages_per_seq > (1 << 24) || num_pages < 1 || num_pages > (1 << 25) - 1)
        return fail(BF1_ERR_UNSUPPORTED, "max_pages_per_seq up to 2^24 and num_pages up to 2^25 - 1");
    const int need = bf1_cache_plan_units(out->batch, out->capacity_tokens);
    if (out->capacity_units < need) return fail(BF1_ERR_CAPACITY, "cache plan capacity_units %d < %d", out->capacity_units, need);
    TableArgs a;
    a.lens = seqlens_dev;
    a.add = new_lens_dev;
    a.table = page_table_dev;
    a.free_pages = free_pages_dev;
    a.free_count = free_count_dev;
    a.batch = out->batch;
    a.max_pages = max_pages_per_seq;
    a.num_pages = num_pages;
    a.p = *out;
    // one CTA for what its threads do in a few rounds
    const int ctas = out->capacity_tokens <= 8192 && out->batch <= kTableThreads ? 1 : 8;
    // us with 128 / 256 / 512 / 1024 threads: 120 sequences of a token 3.6 / 3.7 / 4.1 / 5.2, 26 of 22 4.6 / 4.3 / 4.6 / 5.5, 240 of a token 5.2 / 4.1 /
    // 4.4 / 5.5, of 30 9.6 / 6.5 / 6.2 / 7.1, 600 of a token 10.6 / 7.4 / 6.6 / 6.4
    const int threads = ctas > 1 || out->batch > 512 ? kTableThreads
                        : out->batch > 256 || out->capacity_tokens > 4096 ? 512 : out->batch > 128 || out->capacity_tokens > 512 ? 256 : 128;
    BF1_CUDA_CHECK(launch_pdl_cluster(plan_cache_kernel, dim3(ctas), dim3(ctas), threads, 0, (cudaStream_t)stream, a));
    return BF1_OK;
}

extern "C" int bf1_cache_write(const bf1_rows* k, const bf1_rows* v, const bf1_rows* q, int32_t tokens, int32_t hq, int32_t hkv, int32_t d,
                               const bf1_cache_plan* plan, const bf1_rope* rope, int32_t num_pages, void* k_pages, void* v_pages,
                               float* k_scales, float* v_scales, const bf1_rows* out_q, void* stream) {
    if (int rc = check_plan(plan)) return rc;
    if (tokens < 0 || hkv < 1 || hq < 0 || num_pages < 1) return fail(BF1_ERR_INVALID_ARG, "bad token, head or page count");
    if (d != 64 && d != 128) return fail(BF1_ERR_UNSUPPORTED, "head dimension %d: only 64 and 128 are supported", d);
    if (tokens != plan->capacity_tokens) return fail(BF1_ERR_INVALID_ARG, "%d tokens, the plan is for %d", tokens, plan->capacity_tokens);
    if (hkv > 65535 || hq > 65535) return fail(BF1_ERR_UNSUPPORTED, "%d query and %d KV heads", hq, hkv);
    if (!k_pages || !v_pages) return fail(BF1_ERR_INVALID_ARG, "k_pages or v_pages is null");
    if (((uintptr_t)k_pages | (uintptr_t)v_pages) & 15) return fail(BF1_ERR_INVALID_ARG, "k_pages and v_pages must be 16-byte aligned");
    if ((k_scales == nullptr) != (v_scales == nullptr)) return fail(BF1_ERR_INVALID_ARG, "k_scales and v_scales go together");
    if (hq > 0 && !rope) return fail(BF1_ERR_INVALID_ARG, "queries are there to be rotated: no rope is given");
    if (rope)
        if (int rc = check_rope(rope, d)) return rc;
    if (tokens == 0 || plan->batch == 0) return BF1_OK;
    const bf1_rows* rows[4] = {k, v, q, out_q};
    const char* const names[4] = {"k", "v", "q", "out_q"};
    for (int i = 0; i < (hq ? 4 : 2); ++i)
        if (int rc = check_rows(rows[i], names[i])) return rc;
    if (hq && q->data == out_q->data && (q->row_stride != out_q->row_stride || q->head_stride != out_q->head_stride))
        return fail(BF1_ERR_INVALID_ARG, "out_q in place of q has to have its strides");
    WriteArgs a;
    a.x[0] = rows_of(k);
    a.x[1] = rows_of(v);
    a.q = hq ? rows_of(q) : a.x[0];
    a.out_q = hq ? rows_of(out_q) : a.x[0];
    a.pages[0] = static_cast<uint8_t*>(k_pages);
    a.pages[1] = static_cast<uint8_t*>(v_pages);
    a.scales[0] = k_scales;
    a.scales[1] = v_scales;
    a.units = reinterpret_cast<const int4*>(plan->units);
    a.positions = plan->positions;
    a.status = plan->status;
    a.rope = rope ? table_of(rope) : RopeTable{nullptr, 0, 0, 1.f};
    a.tokens = tokens;
    a.hq = hq;
    a.hkv = hkv;
    a.num_pages = num_pages;
    static const WriteKernel tokens_kernels[2][2][2] = {   // [a rope][8 bits][d = 128]
        {{cache_write_tokens_kernel<64, false, false>, cache_write_tokens_kernel<128, false, false>},
         {cache_write_tokens_kernel<64, true, false>, cache_write_tokens_kernel<128, true, false>}},
        {{cache_write_tokens_kernel<64, false, true>, cache_write_tokens_kernel<128, false, true>},
         {cache_write_tokens_kernel<64, true, true>, cache_write_tokens_kernel<128, true, true>}}};
    static const WriteKernel pages_kernels[2][2][2] = {
        {{cache_write_pages_kernel<64, false>, cache_write_pages_kernel<128, false>}, {cache_write_pages_kernel<64, true>, cache_write_pages_kernel<128, true>}},
        {{cache_write_turned_kernel<64, false>, cache_write_turned_kernel<128, false>}, {cache_write_turned_kernel<64, true>, cache_write_turned_kernel<128, true>}}};
    // Few tokens to a sequence, as far as the host knows: a warp to a unit and head, which shares a CTA's angles with three others.  us, so / a CTA to a unit
    // (16 / 8 heads, d = 128, 8 bits, rotated on the way): 256 sequences of one token 4.0 / 5.7, of two 6.1 / 17.1, of four 15.1 / 22.6, eight of four 6.5 / 4.2,
    // of seven 11.3 / 4.5; 508 of one and four of 120 62 / 32, 480 of one and 32 of 100 177 / 43.
    const bool few = tokens <= 2 * (int64_t)plan->batch, turned = rope != nullptr;
    const int64_t units = bf1_cache_plan_units(plan->batch, tokens);
    if (plan->capacity_units < units) return fail(BF1_ERR_CAPACITY, "cache plan capacity_units %d < %d", plan->capacity_units, (int)units);
    a.num_units = (int32_t)units;
    // heads that share their angles: as many as leave three CTAs for every SM
    a.heads_per_cta = (int)std::max<int64_t>(1, std::min<int64_t>(hkv, units * 2 * hkv / (3 * 148)));
    a.write_ctas = few ? units * ((hkv + 3) / 4) : turned ? units * 2 * ((hkv + a.heads_per_cta - 1) / a.heads_per_cta) : units * 2 * hkv;
    int64_t token_ctas = 0;
    a.q_shares = 0;
    if (hq && few) {
        const int per_cta = d == 128 ? kRopeTokens<128> : kRopeTokens<64>;
        token_ctas = ((int64_t)tokens + per_cta - 1) / per_cta;
        a.q_shares = (int)std::max<int64_t>(1, std::min<int64_t>((hq + 3) / 4, 148 * 8 / token_ctas));
    } else if (hq) {   // a launch of their own: beside the writes they would have those CTAs' registers (18000 tokens of one head 24 us, 22 as it is)
        if (int rc = bf1_rope_fwd(q, nullptr, plan->positions, tokens, hq, 0, d, rope, out_q, nullptr, stream)) return rc;
    }
    const int64_t ctas = a.write_ctas + token_ctas * a.q_shares;
    if (ctas > 0x7fffffffLL) return fail(BF1_ERR_UNSUPPORTED, "%d tokens of %d query and %d KV heads in one call", tokens, hq, hkv);
    BF1_CUDA_CHECK(launch_pdl((few ? tokens_kernels : pages_kernels)[turned][k_scales != nullptr][d == 128], dim3((unsigned)ctas),
                              !few && turned ? kTurnThreads : 128, 0, (cudaStream_t)stream, a));
    return BF1_OK;
}
