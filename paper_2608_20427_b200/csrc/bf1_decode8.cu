// One-token decode over a paged cache in 8 bits: pages of e4m3 numbers, one fp32 scale for each page and KV head.
//
//   o = sum_i p_i sv(i) v_i / sum_i p_i,   p_i = exp(scale * sk(i) <q, k_i>),   i over the keys of the plan's pages
//
// Every key costs 2 d bytes and 4 d G operations: bound by HBM for as long as the arithmetic on a page (16 KB of K and V at
// d = 128) stays hidden behind the copies, 700 cycles of an SM.  Short lists are walked by a CTA each, or by a cluster whose CTAs exchange their parts (max,
// sum, O) through shared memory.  The list of a dense layer has hundreds of pages, and lists are of all lengths: then the work is not dealt by lists, but for
// every KV head the pages of all of them stand in one row, which is cut into equal runs, one to a CTA, as many as the SMs hold at once.  The CTAs that read
// the heads of one page run side by side, so that its rows are fetched together.  A list that a cut goes through is left as partial results, which a second
// small kernel adds up in list order.  Measured: 24 lists of up to 32K tokens, 16 query / 8 KV heads, d = 128, 842 MB: 131 to 132 us, 6.4 TB/s, 98 to 99 % of
// a copy's rate; one sequence of 100K tokens 40.4 us (floor 31.7), 32 along the route 12.5 (7.2), one along the route 4.2.
//
// In a CTA one warp asks for pages by TMA into a ring, and four warps take 16 keys of every page each.  The numbers of the cache are the A
// operand of m16n8k16 (16 keys or 16 dimensions to a row, the heads are the eight columns): widened from e4m3 to f16, which is
// exact, two at a time.  q, eight significant bits in bf16, is exact in f16 too, down to 2^-31 of the head's largest value, once it is scaled to that; P in f16 is rounded
// by 2^-11, an eighth of what bf16 would cost.  So that this holds for small weights too, P is made against the largest of the sixteen keys (not of the list) and
// enters times 2^15: f16 has all its digits down to 2^-29 of that one, and steps of 2^-39 of it below.  (Against the list's largest and times 1, a key 17 nats
// above the others took all weight from those that its warp saw: with a value of zero it left nothing but rounding.)  Scales stay outside of the
// products, in 32 bits: sk on the scores, sv on each page's sum, together with the weight of the sixteen keys' largest in the list.
#include <math.h>

#include <algorithm>
#include <atomic>
#include <cfloat>
#include <cuda.h>

#include "bf1_common.cuh"

namespace bf1 {

constexpr int kP8 = 64;                  // tokens per page
constexpr int kD8Consumers = 128, kD8Threads = kD8Consumers + 32;
constexpr int kD8MaxStages = 8;
constexpr int kD8MaxScan = 1024;         // sequences whose lists are cut (more of them: a CTA per list)
constexpr int kD8MaxRuns = 640;          // runs at most, which is what the workspace has room for
constexpr int kD8MinRun = 4;             // pages of a run at least
constexpr int kD8MaxCtas = 16;           // to a cluster
constexpr int kD8Held = 64;              // pages of a list that the copying warp holds at once
constexpr float kPUp = 32768.f;          // P enters the products times 2^15, so that f16 has eleven digits of it down to 2^-29

// How the lists are dealt: kRuns as above; kWhole a CTA per list; kParts a cluster per list, each CTA an even part of it.
enum { kRuns, kWhole, kParts };

struct Decode8Args {
    const __nv_bfloat16* q;              // [rows, hq, d]
    const float *k_scales, *v_scales;    // [pages, hkv]
    const int32_t *seqlens, *count, *page, *block;
    const int32_t* cu_tokens;            // [batch + 1] the sequences' new tokens among the rows, or null: row s is sequence s
    int32_t* status;
    int32_t rows;                        // of q, o and lse
    int32_t max_degree, hq, hkv, num_pages, group, batch;
    float scale_log2;
    __nv_bfloat16* o;                    // [rows, hq, d]
    float* lse;                          // [hq, rows]
    int32_t runs;                        // kRuns: per KV head
    int32_t stages, ahead;               // pages in a CTA's ring, and of those asked for at once at the start
    int32_t nctas, share;                // kParts: CTAs to a list, columns (of the heads' G d) that each adds up, a multiple of 32
    int32_t* bases;                      // workspace: [batch + 2] pages in front of every list, runs in use
    float2* part_ml;                     // [hkv][runs][2][group] (max, sum) ...
    float* part_o;                       // [hkv][runs][2][group][d] ... and sum of a cut list's part
};

// Runs that a row of `pages` pages is cut into: of kD8MinRun pages at least, so that short rows are not all joining (and none is empty), and so that the
// longest list, of `longest` pages, is cut into no more than four times the root of that: a page more to a run costs what the join of its part would (0.4 us,
// and 0.03 for each part).
__device__ __forceinline__ int runs_of(int runs, long long pages, int longest) {
    const long long most = (pages + kD8MinRun - 1) / kD8MinRun;
    return (int)fminf((float)min((long long)runs, most), ceilf(4.f * (float)pages * rsqrtf((float)max(longest, 1))));
}

// The row of a sequence's newest token; within the arrays whatever stands there by now (pages_of_list has refused others).
__device__ __forceinline__ int row_of_list(const Decode8Args& a, int s) {
    return a.cu_tokens ? min(max(a.cu_tokens[s + 1] - 1, 0), a.rows - 1) : s;
}

// A launch on this status word has given up a wait: nothing is done until a plan clears it.
__device__ __forceinline__ bool given_up(const Decode8Args& a) { return *a.status & BF1_DEV_WAIT_TIMEOUT; }

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* tmap, int c0, int c1, int c2, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
        "[%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
// Two e4m3 numbers of the low / high half of a word as f16x2.
__device__ __forceinline__ uint32_t widen_lo(uint32_t v) {
    uint32_t r;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\t}" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t widen_hi(uint32_t v) {
    uint32_t r;
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, b;\n\t}" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kD8Consumers) : "memory"); }

// The 16-byte chunk `c` of row r of a page in shared memory, rows of D bytes, as TMA swizzles them (128 B or 64 B).
template <int D>
__device__ __forceinline__ uint32_t page_chunk(int r, int c) {
    return r * D + ((c ^ (D == 128 ? r & 7 : (r >> 1) & 3)) << 4);
}

// The queries of a list's heads as the B operand of the scores: column gid is head gid, and the four values that a lane holds of
// chunk c are the dimensions 16 c + 4 tig .. + 3, the order in which ldmatrix hands out K's bytes.  Scaled by a power of two that puts the
// head's largest value into [2^14, 2^15): what is above 2^-31 of it has all its digits, and what is
// below half of 2^-38 is zero.  f[0], f[1]: what the scores of heads 2 tig and
// 2 tig + 1 have to be multiplied with (the softmax's scale and log2 e in it).
template <int D>
__device__ __forceinline__ void load_queries(const Decode8Args& a, int row, int hbase, uint32_t (&qb)[D / 16][2], float (&f)[2]) {
    const int lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    float x[D / 16][4], top = 0.f;
    const uint2* head = reinterpret_cast<const uint2*>(a.q + ((size_t)row * a.hq + hbase + (gid < a.group ? gid : 0)) * D);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
        const uint2 v = gid < a.group ? head[c * 4 + tig] : make_uint2(0u, 0u);
        x[c][0] = __uint_as_float(v.x << 16);
        x[c][1] = __uint_as_float(v.x & 0xffff0000u);
        x[c][2] = __uint_as_float(v.y << 16);
        x[c][3] = __uint_as_float(v.y & 0xffff0000u);
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, fabsf(x[c][i]));
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int e = max((int)(__float_as_uint(top) >> 23) - 127, -100);              // 128 if it is infinite
    const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);              // 2^(14 - e)
    const float down = a.scale_log2 * __uint_as_float((uint32_t)(127 - 14 + e) << 23);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
        qb[c][0] = pack_f16x2(x[c][0] * up, x[c][1] * up);
        qb[c][1] = pack_f16x2(x[c][2] * up, x[c][3] * up);
    }
    f[0] = __shfl_sync(0xffffffffu, down, 8 * tig);                                // lanes 4 h hold head h
    f[1] = __shfl_sync(0xffffffffu, down, 8 * tig + 4);
}

// One warp's softmax over the keys it has seen: lanes hold heads 2 tig and 2 tig + 1.
template <int D>
struct WarpState {
    float m[2], l[2];
    uint64_t acc[D / 16][2];             // acc[c][i]: dimension 16 c + 2 gid + i of the two heads, side by side
    __device__ __forceinline__ void clear() {
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.f;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) acc[c][0] = acc[c][1] = 0ull;
    }
};

// Keys key0 .. key0 + 15 of kPages pages in shared memory (K, and V behind it), of which the first `valid` of the last page count.
// Two pages at a time: their chains of dependent products run side by side.
template <int D, int kPages>
__device__ __forceinline__ void page_step(WarpState<D>& w, const uint32_t (&kb)[kPages], int key0, int valid, const uint32_t (&qb)[D / 16][2],
                                          const float (&f)[2], const float2 (&scales)[kPages]) {
    const int lane = threadIdx.x & 31, gid = lane >> 2;
    const int row = key0 + (lane & 15), odd = lane >> 4;     // ldmatrix: keys 0-7 and 8-15 of one chunk, then of the next
    if (valid < key0 + 16) {                                 // rows behind the newest token may hold anything, NaN included
        const uint32_t vb = kb[kPages - 1] + kP8 * D;
        for (int i = lane; i < 16 * (D / 16); i += 32)
            if (key0 + i / (D / 16) >= valid) st_shared_v4(vb + (key0 + i / (D / 16)) * D + i % (D / 16) * 16, 0u, 0u, 0u, 0u);
        fence_proxy_async();                                 // (the next copy into this place comes behind these)
        __syncwarp();
    }
    float sc[kPages][4], sd[kPages][4];                      // even and odd chunks for themselves
#pragma unroll
    for (int p = 0; p < kPages; ++p)
#pragma unroll
        for (int i = 0; i < 4; ++i) sc[p][i] = sd[p][i] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 16; c += 2)
#pragma unroll
        for (int p = 0; p < kPages; ++p) {
            uint32_t r[4];
            ldsm4(kb[p] + page_chunk<D>(row, c + odd), r);
            mma_f16(sc[p], widen_lo(r[0]), widen_lo(r[1]), widen_hi(r[0]), widen_hi(r[1]), qb[c][0], qb[c][1]);
            mma_f16(sd[p], widen_lo(r[2]), widen_lo(r[3]), widen_hi(r[2]), widen_hi(r[3]), qb[c + 1][0], qb[c + 1][1]);
        }
    uint32_t v[kPages][D / 32][4];                           // V is on its way to registers while the softmax is made
#pragma unroll
    for (int c = 0; c < D / 16; c += 2)
#pragma unroll
        for (int p = 0; p < kPages; ++p) ldsm4_trans(kb[p] + kP8 * D + page_chunk<D>(row, c + odd), v[p][c / 2]);
    // keys gid (0, 1) and gid + 8 (2, 3) of heads 2 tig and 2 tig + 1
    float mx[kPages][2], al[2], base[2], by[kPages][2];
#pragma unroll
    for (int p = 0; p < kPages; ++p)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float to = f[h] * scales[p].x;
            const int there = p == kPages - 1 ? valid : kP8;
            sc[p][h] = key0 + gid < there ? (sc[p][h] + sd[p][h]) * to : -INFINITY;
            sc[p][2 + h] = key0 + gid + 8 < there ? (sc[p][2 + h] + sd[p][2 + h]) * to : -INFINITY;
            mx[p][h] = fmaxf(sc[p][h], sc[p][2 + h]);
        }
#pragma unroll
    for (int off = 4; off < 32; off <<= 1)
#pragma unroll
        for (int p = 0; p < kPages; ++p)
#pragma unroll
            for (int h = 0; h < 2; ++h) mx[p][h] = fmaxf(mx[p][h], __shfl_xor_sync(0xffffffffu, mx[p][h], off));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float m = w.m[h];
#pragma unroll
        for (int p = 0; p < kPages; ++p) m = fmaxf(m, mx[p][h]);
        base[h] = m == -INFINITY ? 0.f : m;                  // (scores of minus infinity alone)
        al[h] = ex2_approx(w.m[h] - base[h]);
        w.m[h] = m;
        w.l[h] *= al[h];
#pragma unroll
        for (int p = 0; p < kPages; ++p) {                   // weights against the sixteen keys' own largest, which `by` brings to the list's
            const float own = mx[p][h] == -INFINITY ? 0.f : mx[p][h];
            sc[p][h] = ex2_approx(sc[p][h] - own);
            sc[p][2 + h] = ex2_approx(sc[p][2 + h] - own);
            by[p][h] = ex2_approx(mx[p][h] - base[h]);       // 0 where no key counts
            w.l[h] = fmaf(by[p][h], sc[p][h] + sc[p][2 + h], w.l[h]);
            sc[p][h] *= kPUp;
            sc[p][2 + h] *= kPUp;
            by[p][h] *= scales[p].y * (1.f / kPUp);
        }
    }
    const bool rescale = __any_sync(0xffffffffu, al[0] != 1.f || al[1] != 1.f);
    uint32_t b[kPages][2];
#pragma unroll
    for (int p = 0; p < kPages; ++p) {
        b[p][0] = transpose8x8(pack_f16x2(sc[p][0], sc[p][1]));
        b[p][1] = transpose8x8(pack_f16x2(sc[p][2], sc[p][3]));
    }
    const uint64_t al2 = pack2(al[0], al[1]);
#pragma unroll
    for (int c = 0; c < D / 16; c += 2) {
        if (rescale) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 2; ++i) w.acc[c + u][i] = mul2(w.acc[c + u][i], al2);
        }
#pragma unroll
        for (int p = 0; p < kPages; ++p) {
            uint32_t r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = __byte_perm(v[p][c / 2][i], 0, 0x3120);     // (two keys of one dimension side by side)
            const uint64_t by2 = pack2(by[p][0], by[p][1]);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                float pa[4] = {0.f, 0.f, 0.f, 0.f};
                mma_f16(pa, widen_lo(r[2 * u]), widen_hi(r[2 * u]), widen_lo(r[2 * u + 1]), widen_hi(r[2 * u + 1]), b[p][0], b[p][1]);
#pragma unroll
                for (int i = 0; i < 2; ++i) w.acc[c + u][i] = fma2(by2, pack2(pa[2 * i], pa[2 * i + 1]), w.acc[c + u][i]);
            }
        }
    }
}

template <int D, int kHeads>
struct Merge8 {                          // the four warps' states at the end of a list or a part of it
    float o[4][kHeads][D + 4], m[4][kHeads], l[4][kHeads];
};

// grid (hkv, runs), (hkv, batch) or (hkv, batch, CTAs of the cluster)
template <int D, int kHeads, int kMode>
__global__ void __launch_bounds__(kD8Threads, kMode == kWhole && D == 64 ? 4 : 3) decode8_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                                                                const Decode8Args a) {
    constexpr int kPageBytes = kP8 * D;
    extern __shared__ uint8_t dsmem[];
    __shared__ uint64_t bars[2 * kD8MaxStages];
    __shared__ float2 page_scales[kD8MaxStages];
    __shared__ Merge8<D, kHeads> st;
    __shared__ int warp_sums[kD8Threads / 32], warp_most[kD8Threads / 32];
    __shared__ int abort_flag, list_count;
    const uint32_t ring = (smem_u32(dsmem) + 1023) & ~1023u;
    uint8_t* const behind = dsmem + (ring - smem_u32(dsmem)) + (size_t)a.stages * 2 * kPageBytes;
    int* const bases = reinterpret_cast<int*>(behind);                 // kRuns
    const uint32_t sums_at = smem_u32(behind), gather_at = sums_at + (a.nctas * kHeads * 8 + 15) / 16 * 16;   // kParts: [CTA][head] (max, sum), [CTA][share] columns
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, kvh = blockIdx.x;
    const uint32_t full = smem_u32(bars), empty = full + 8 * kD8MaxStages;
    if (tid == 0) {
        abort_flag = 0;
        for (int i = 0; i < a.stages; ++i) {
            mbar_init(full + 8 * i, 2);                               // the copies, the scales
            mbar_init(empty + 8 * i, kD8Consumers / 32);
        }
        fence_mbar_init();
        tma_prefetch_desc(&tm_k);
        tma_prefetch_desc(&tm_v);
    }
    pdl_wait();
    const bool reports = kvh == 0 && blockIdx.z == 0;
    auto pages_of_list = [&](int s, bool report) {
        const int n = a.seqlens[s];
        int c = max(min(a.count[s], a.max_degree), 0);
        if (a.cu_tokens) {                                           // a sequence without a token in this step has no row
            const int first = a.cu_tokens[s], end = a.cu_tokens[s + 1];
            if (end <= first) c = 0;
            else if (first < 0 || end > a.rows) {
                if (c > 0 && report) atomicOr(a.status, BF1_DEV_BAD_ROUTE);
                c = 0;
            }
        }
        if (c > 0 && (n < 1 || (n - 1) / kP8 != a.block[s])) {       // the plan belongs to another 64 tokens
            if (report) atomicOr(a.status, BF1_DEV_BAD_ROUTE);
            return 0;
        }
        return c;
    };
    // ---- this CTA's pages: x0 .. x1 - 1 of the row (kRuns), or of its list -------------------------------------------------------------
    int s = 0, x0 = 0, x1 = 0, count = 0, held[2] = {-1, -1};
    bool dead = false;                                               // nothing may be written of this list
    if constexpr (kMode != kRuns) {
        s = blockIdx.y;
        if (warp == kD8Consumers / 32)                               // the list is asked for together with its length
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (lane + 32 * i < a.max_degree) held[i] = a.page[(size_t)s * a.max_degree + lane + 32 * i];
        // read once, since threads that disagreed would not meet at the barriers, and not by the thread that sets these up
        if (tid == 32) {
            const bool stopped = given_up(a);                        // (asked for with the length, not in front of it)
            const int c = pages_of_list(s, reports);
            list_count = stopped ? -1 : c;
        }
        __syncthreads();                                             // the barriers are there
        dead = list_count < 0;
        count = max(list_count, 0);
        x0 = kMode == kParts ? blockIdx.z * count / a.nctas : 0;
        x1 = kMode == kParts ? (blockIdx.z + 1) * count / a.nctas : count;
        if (kMode == kWhole && count == 0) return;
        if constexpr (kMode == kParts) cluster_arrive_relaxed();     // (waited for in front of the first store to another CTA)
    } else {
        const int per = (a.batch + kD8Threads - 1) / kD8Threads, lo = min(tid * per, a.batch), hi = min(lo + per, a.batch);
        if (tid == kD8Threads - 1) list_count = given_up(a) ? -1 : 0;        // (by a warp that has nothing to look up here unless lists are many)
        int sum = 0, longest = 0;
        for (int i = lo; i < hi; ++i) {
            const int c = pages_of_list(i, kvh == 0 && blockIdx.y == 0);
            bases[i] = c;
            sum += c;
            longest = max(longest, c);
        }
        int incl = sum;
        longest = __reduce_max_sync(0xffffffffu, longest);
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl += v;
        }
        if (lane == 31) warp_sums[warp] = incl, warp_most[warp] = longest;
        __syncthreads();
        int at = incl - sum;
        for (int w = 0; w < warp; ++w) at += warp_sums[w];
#pragma unroll
        for (int w = 0; w < kD8Threads / 32; ++w) longest = max(longest, warp_most[w]);
        for (int i = lo; i < hi; ++i) {
            const int c = bases[i];
            bases[i] = at;
            at += c;
        }
        if (lo < hi && hi == a.batch) bases[a.batch] = at;
        __syncthreads();
        const long long total = bases[a.batch];
        const int runs = runs_of(a.runs, total, longest);
        if ((int)blockIdx.y < runs && total > 0 && list_count == 0) {
            x0 = (int)(total * blockIdx.y / runs);
            x1 = (int)(total * (blockIdx.y + 1) / runs);
        }
        if (kvh == 0 && blockIdx.y == 0)
            for (int i = tid; i <= a.batch + 1; i += kD8Threads) a.bases[i] = i <= a.batch ? bases[i] : runs;
        if (x0 >= x1) return;
    }
    // the list that page x belongs to
    auto list_of = [&](int x) {
        if constexpr (kMode != kRuns) return s;
        int lo = 0, hi = a.batch;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (bases[mid] <= x) lo = mid;
            else hi = mid;
        }
        return lo;
    };
    if (warp == kD8Consumers / 32) {
        // ---- the copying warp: a lane looks up a page, 32 pages ahead of their use -----------------------------------------------------
        auto look_up = [&](int x) {
            int pg = 0;
            if constexpr (kMode != kRuns) {
                const int h0 = __shfl_sync(0xffffffffu, held[0], x & 31), h1 = __shfl_sync(0xffffffffu, held[1], x & 31);
                pg = x < 32 ? h0 : h1;
            }
            if (x >= x1) return 0;
            if (kMode == kRuns || x >= kD8Held) {
                const int sx = list_of(x);
                pg = a.page[(size_t)sx * a.max_degree + (kMode == kRuns ? x - bases[sx] : x)];
            }
            if (pg < 0 || pg >= a.num_pages) {
                atomicOr(a.status, BF1_DEV_BAD_ROUTE);
                pg = 0;
            }
            return pg;
        };
        auto scales_of = [&](int x, int pg) {
            return x < x1 ? make_float2(a.k_scales[(size_t)pg * a.hkv + kvh], a.v_scales[(size_t)pg * a.hkv + kvh]) : make_float2(0.f, 0.f);
        };
        auto copy = [&](int to_stage, int pg) {
            const uint32_t bar = full + 8 * to_stage, to = ring + to_stage * 2 * kPageBytes;
            mbar_expect_tx(bar, 2 * kPageBytes);
            tma_load_3d(to, &tm_k, 0, kvh, pg * kP8, bar);
            tma_load_3d(to + kPageBytes, &tm_v, 0, kvh, pg * kP8, bar);
        };
        int pg = look_up(x0 + lane), stage = 0, parity = 1, issued = 0;
        // the ring is empty: its first pages are asked for while the scales are still being fetched
        const int ahead = min(x1 - x0, min(a.ahead, a.stages));
        for (int i = 0; i < ahead; ++i) {
            const int p = __shfl_sync(0xffffffffu, pg, i);
            if (elect_one()) copy(i, p);
            __syncwarp();
        }
        float2 sc = scales_of(x0 + lane, pg);
        bool ok = true;
        for (int xb = x0; xb < x1 && ok; xb += 32) {
            const int pg_next = look_up(xb + 32 + lane);
            const float2 sc_next = scales_of(xb + 32 + lane, pg_next);
            const int n = min(32, x1 - xb);
            for (int i = 0; i < n; ++i) {
                const int p = __shfl_sync(0xffffffffu, pg, i);
                const float2 ps = make_float2(__shfl_sync(0xffffffffu, sc.x, i), __shfl_sync(0xffffffffu, sc.y, i));
                if (issued >= ahead) {
                    const uint32_t bar = issued >= a.stages ? empty + 8 * stage : full + 8 * (issued - ahead);
                    ok = __all_sync(0xffffffffu, mbar_wait(bar, issued >= a.stages ? parity : 0, &abort_flag, a.status));
                    if (!ok) break;
                }
                if (lane == 0) {
                    if (issued >= ahead) copy(stage, p);
                    page_scales[stage] = ps;
                    mbar_arrive(full + 8 * stage);
                }
                __syncwarp();
                ++issued;
                if (++stage == a.stages) stage = 0, parity ^= 1;
            }
            pg = pg_next;
            sc = sc_next;
        }
        if (!ok) {                                           // given up: the copies on their way have to land all the same
            const long long t0 = clock64();
            for (int i = max(0, issued - a.stages); i < issued; ++i)
                while (!mbar_try_wait(full + 8 * (i % a.stages), i / a.stages & 1) && clock64() - t0 < kWaitCycles) {
                }
        }
        if constexpr (kMode == kParts) {                     // (the whole CTA arrives at the cluster's barriers)
            __syncwarp();
            cluster_wait();
            cluster_arrive();
            cluster_wait();
        }
        return;
    }
    // ---- the four warps that compute: one list, or the part of it that lies in this run, after the other ----------------------------------
    const int key0 = warp * 16, hbase = kvh * a.group, gid = lane >> 2, tig = lane & 3;
    constexpr int kCols = kHeads * D / kD8Consumers, kPerHead = kD8Consumers / kHeads;
    const int h = tid / kPerHead, c0 = tid % kPerHead * kCols;
    int stage = 0, parity = 0, row = 0;
    s = list_of(x0);
    if constexpr (kMode != kRuns) row = row_of_list(a, s);
    // the part of list s from page x to `end` (of `last`), and the four warps' states merged: (max, sum) and this thread's columns
    auto part = [&](int x, int end, int last, float& m, float& l, float (&out)[kCols]) {
        const int n = a.seqlens[s], tail = n - (n - 1) / kP8 * kP8;
        if constexpr (kMode == kRuns) row = row_of_list(a, s);
        uint32_t qb[D / 16][2];
        float f[2];
        load_queries<D>(a, row, hbase, qb, f);
        WarpState<D> w;
        w.clear();
        auto next = [&]() {                                  // waits for a page; its place in the ring
            mbar_wait(full + 8 * stage, parity, &abort_flag, a.status);
            const int at = stage;
            if (++stage == a.stages) stage = 0, parity ^= 1;
            return at;
        };
        // (a run's ring of three pages of d = 128 would have one on its way while two are taken)
        for (; (kMode != kRuns || D == 64) && x + 1 < end && a.stages > 1; x += 2) {
            const int p0 = next(), p1 = next();
            const uint32_t kb[2] = {ring + p0 * 2 * kPageBytes, ring + p1 * 2 * kPageBytes};
            const float2 scales[2] = {page_scales[p0], page_scales[p1]};
            page_step<D, 2>(w, kb, key0, x + 1 == last - 1 ? tail : kP8, qb, f, scales);
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(empty + 8 * p0);
                mbar_arrive(empty + 8 * p1);
            }
        }
        for (; x < end; ++x) {
            const int p0 = next(), valid = x == last - 1 ? tail : kP8;
            const uint32_t kb[1] = {ring + p0 * 2 * kPageBytes};
            const float2 scales[1] = {page_scales[p0]};
            if (key0 < valid) page_step<D, 1>(w, kb, key0, valid, qb, f, scales);
            __syncwarp();
            if (lane == 0) mbar_arrive(empty + 8 * p0);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) w.l[i] += __shfl_xor_sync(0xffffffffu, w.l[i], off);
        if (2 * tig < kHeads) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (gid == 0) {
                    st.m[warp][2 * tig + i] = w.m[i];
                    st.l[warp][2 * tig + i] = w.l[i];
                }
            }
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                float even[2], odd[2];
                unpack2(w.acc[c][0], even[0], even[1]);
                unpack2(w.acc[c][1], odd[0], odd[1]);
#pragma unroll
                for (int i = 0; i < 2; ++i) *reinterpret_cast<float2*>(&st.o[warp][2 * tig + i][16 * c + 2 * gid]) = make_float2(even[i], odd[i]);
            }
        }
        consumers_sync();
        m = fmaxf(fmaxf(st.m[0][h], st.m[1][h]), fmaxf(st.m[2][h], st.m[3][h]));
        const float base = m == -INFINITY ? 0.f : m;
        l = 0.f;
#pragma unroll
        for (int c = 0; c < kCols; ++c) out[c] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float by = exp2f(st.m[i][h] - base);       // 0 for a warp that has seen no key
            l = fmaf(by, st.l[i][h], l);
#pragma unroll
            for (int c = 0; c < kCols; ++c) out[c] = fmaf(by, st.o[i][h][c0 + c], out[c]);
        }
    };
    // (read behind a barrier of the four warps that part() ends with: all of them see what one of them, or the copying warp it waited for, has set)
    auto gave_up = [&]() { return *const_cast<const volatile int*>(&abort_flag) != 0; };
    auto write = [&](float m, float l, const float (&out)[kCols]) {
        if (h >= a.group || gave_up()) return;               // G = 1: the second head does not exist
        const float inv = 1.f / l;
        __nv_bfloat16* orow = a.o + ((size_t)row * a.hq + hbase + h) * D + c0;
#pragma unroll
        for (int c = 0; c < kCols; ++c) orow[c] = __float2bfloat16_rn(out[c] * inv);
        if (c0 == 0) a.lse[(size_t)(hbase + h) * a.rows + row] = (m + log2f(l)) * 0.6931471805599453f;
    };
    float m, l, out[kCols];
    if constexpr (kMode == kWhole) {
        part(0, x1, x1, m, l, out);
        write(m, l, out);
    } else if constexpr (kMode == kRuns) {
        for (int x = x0; x < x1;) {
            while (bases[s + 1] <= x) ++s;                   // (empty lists)
            const int first = bases[s], last = bases[s + 1], end = min(x1, last);
            part(x - first, end - first, last - first, m, l, out);
            if (x == first && end == last) {
                write(m, l, out);
            } else if (h < a.group && !gave_up()) {          // (the join does not read them then)
                // a run cuts at most two lists: the one it begins in and the one it ends in
                const size_t slot = (((size_t)kvh * a.runs + blockIdx.y) * 2 + (x == first ? 1 : 0)) * a.group + h;
#pragma unroll
                for (int c = 0; c < kCols; ++c) a.part_o[slot * D + c0 + c] = out[c];
                if (c0 == 0) a.part_ml[slot] = make_float2(m, l);
            }
            x = end;
            consumers_sync();                                // (the states are written again)
        }
    } else {
        if (x0 < x1) {
            part(x0, x1, count, m, l, out);
            if (gave_up()) m = NAN;                          // (a maximum is never NaN: it tells the others)
        } else {                                             // zeros, under a weight of zero
            m = dead ? NAN : -INFINITY;
            l = 0.f;
#pragma unroll
            for (int c = 0; c < kCols; ++c) out[c] = 0.f;
        }
        // ---- the parts of a list are added up in list order: every CTA of the cluster its share of the columns, 32 to a warp, and every
        //      warp the maxima and sums of its head, a part to a lane
        __syncwarp();
        cluster_wait();                                      // the other CTAs of the cluster have started
        {
            const int v = h * D + c0, rank = v / a.share;
            st_cluster(map_cluster(gather_at + (blockIdx.z * a.share + v - rank * a.share) * 4, rank), out);
        }
        if (tid % kPerHead < a.nctas) {
            const float ml[2] = {m, l};
            st_cluster(map_cluster(sums_at + (blockIdx.z * kHeads + h) * 8, tid % kPerHead), ml);
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();                                      // everything for this CTA is in its shared memory
        const int v0 = blockIdx.z * a.share, v_end = count > 0 ? min(v0 + a.share, kHeads * D) : 0;
        for (int v = v0 + tid; v < v_end; v += kD8Consumers) {
            const int hv = v / D, col = v % D;               // (v - lane is a multiple of 32: the same head in a warp)
            const float2* sums = reinterpret_cast<const float2*>(behind) + hv;                                       // [CTA][kHeads]
            const float* parts = reinterpret_cast<const float*>(behind + (gather_at - sums_at)) + (v - v0);           // [CTA][share]
            const float2 ml = lane < a.nctas ? sums[lane * kHeads] : make_float2(-INFINITY, 0.f);
            if (__any_sync(0xffffffffu, ml.x != ml.x)) continue;              // a part is missing
            float top = ml.x;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            const float w = exp2f(ml.x - (top == -INFINITY ? 0.f : top));     // 0 for a part without entries
            float sum = w * ml.y;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            float o = 0.f;
#pragma unroll
            for (int i0 = 0; i0 < kD8MaxCtas; i0 += 4) {     // four at a time, asked for together
                if (i0 >= a.nctas) break;
                float wi[4], p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    wi[i] = __shfl_sync(0xffffffffu, w, i0 + i);
                    p[i] = parts[min(i0 + i, a.nctas - 1) * a.share];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i0 + i < a.nctas) o = fmaf(wi[i], p[i], o);
            }
            if (hv < a.group) {
                a.o[((size_t)row * a.hq + hbase + hv) * D + col] = __float2bfloat16_rn(o * (1.f / sum));
                if (col == 0) a.lse[(size_t)(hbase + hv) * a.rows + row] = (top + log2f(sum)) * 0.6931471805599453f;
            }
        }
    }
}

// Adds up the lists that cuts go through: a CTA per list and KV head, parts in list order, run by run.  The parts' weights first, a
// thread to each, so that their (max, sum) are asked for at once, as the sums are after that (one after the other was 20 us for 55 parts).
// A CTA has 32 of the columns (four numbers each), so that up to 64 parts are one round of loads.
constexpr int kJoinThreads = 256, kJoinColumns = 32;
template <int D>
__global__ void __launch_bounds__(kJoinThreads) decode8_join_kernel(const Decode8Args a) {
    constexpr int kVec = D / 4;                              // threads to a head's row, 4 columns each
    __shared__ float4 sums[kJoinThreads];
    __shared__ float weights[kD8MaxRuns * 4];                // [part][head]
    __shared__ float tops[kJoinThreads / 32][4], ls[kJoinThreads / 32][4];
    pdl_wait();
    const int kvh = blockIdx.x, s = blockIdx.y, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const bool stopped = given_up(a);                        // (needed in front of the store only: unlike the bases it comes from memory)
    const long long total = a.bases[a.batch], first = a.bases[s], last = a.bases[s + 1];
    if (first == last) return;
    const long long runs = a.bases[a.batch + 1];
    auto run_of = [&](long long x) { return (int)(((x + 1) * runs - 1) / total); };   // the last run that begins at or in front of page x
    const int j0 = run_of(first), j1 = run_of(last - 1), parts = j1 - j0 + 1;
    if (parts == 1) return;                                  // whole: written already
    const int row = row_of_list(a, s);
    auto slot = [&](int j) { return (((size_t)kvh * a.runs + j) * 2 + (j == j0 ? 1 : 0)) * a.group; };
    const int columns = min(a.group * kVec, kJoinColumns), groups = kJoinThreads / columns;
    const int g = tid / columns, column = blockIdx.z * columns + tid % columns, h = column / kVec, c = column % kVec;
    constexpr int kAhead = 8;
    float4 v[kAhead];                                        // this thread's columns of every groups-th part, the first ones asked for now
    auto fetch = [&](int i0) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i0 + u * groups < parts) v[u] = *reinterpret_cast<const float4*>(a.part_o + (slot(j0 + i0 + u * groups) + h) * D + 4 * c);
    };
    fetch(g);
    // (tid % group is the same head in every round: 256 is a multiple of the group)
    const int gh = tid % a.group;
    float top = -INFINITY;
    for (int i = tid; i < parts * a.group; i += kJoinThreads) top = fmaxf(top, a.part_ml[slot(j0 + i / a.group) + gh].x);
#pragma unroll
    for (int off = 16; off >= 4; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    for (int off = 2; off >= a.group; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    if (lane < a.group) tops[warp][lane] = top;
    __syncthreads();
    top = tops[0][gh];
#pragma unroll
    for (int i = 1; i < kJoinThreads / 32; ++i) top = fmaxf(top, tops[i][gh]);
    const float base = top == -INFINITY ? 0.f : top;
    float l = 0.f;
    for (int i = tid; i < parts * a.group; i += kJoinThreads) {
        const float2 ml = a.part_ml[slot(j0 + i / a.group) + gh];
        const float by = exp2f(ml.x - base);
        weights[i] = by;
        l = fmaf(by, ml.y, l);
    }
#pragma unroll
    for (int off = 16; off >= 4; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
    for (int off = 2; off >= a.group; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
    if (lane < a.group) ls[warp][lane] = l;
    __syncthreads();
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = g; i0 < parts; i0 += kAhead * groups) {
        if (i0 != g) fetch(i0);
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (i0 + u * groups < parts) {
                const float by = weights[(i0 + u * groups) * a.group + h];
                o.x = fmaf(by, v[u].x, o.x), o.y = fmaf(by, v[u].y, o.y), o.z = fmaf(by, v[u].z, o.z), o.w = fmaf(by, v[u].w, o.w);
            }
    }
    sums[tid] = o;
    __syncthreads();
    if (g > 0 || stopped) return;
    for (int i = 1; i < groups; ++i) {
        const float4 v = sums[i * columns + tid];
        o.x += v.x, o.y += v.y, o.z += v.z, o.w += v.w;
    }
    float m = tops[0][h];
    l = ls[0][h];
#pragma unroll
    for (int i = 1; i < kJoinThreads / 32; ++i) m = fmaxf(m, tops[i][h]), l += ls[i][h];
    const float inv = 1.f / l;
    *reinterpret_cast<uint2*>(a.o + ((size_t)row * a.hq + kvh * a.group + h) * D + 4 * c) = make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
    if (c == 0) a.lse[(size_t)(kvh * a.group + h) * a.rows + row] = (m + log2f(l)) * 0.6931471805599453f;
}

int make_page_map(CUtensorMap* m, const void* ptr, int64_t pages, int hkv, int d);   // bf1_attn.cu

typedef void (*Decode8Kernel)(CUtensorMap, CUtensorMap, Decode8Args);
struct Decode8Variant {
    Decode8Kernel by_mode[3];            // kRuns, kWhole, kParts
};
template <int D, int kHeads>
static Decode8Variant decode8_variant() {
    return {{decode8_kernel<D, kHeads, kRuns>, decode8_kernel<D, kHeads, kWhole>, decode8_kernel<D, kHeads, kParts>}};
}

// Clusters of `ctas` CTAs of a kernel that the GPU runs at once; asked for once per device and shape.
static int clusters8_that_fit(Decode8Kernel kernel, int dev, int which, int ctas, int stages, size_t smem, int* fit) {
    static std::atomic<int> known[64][4][kD8MaxCtas + 1][kD8MaxStages + 1];   // 0: not asked yet, else one more
    std::atomic<int>& k = known[dev][which][ctas][stages];
    int n = k.load(std::memory_order_relaxed) - 1;
    if (n < 0) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(1, 1, ctas);
        cfg.blockDim = dim3(kD8Threads);
        cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute attr = {};
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = attr.val.clusterDim.y = 1;
        attr.val.clusterDim.z = ctas;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        BF1_CUDA_CHECK(cudaOccupancyMaxActiveClusters(&n, kernel, &cfg));
        k.store(n + 1, std::memory_order_relaxed);
    }
    *fit = n;
    return BF1_OK;
}
static size_t up16(size_t x) { return (x + 15) / 16 * 16; }

}  // namespace bf1

using namespace bf1;

// [bases | (max, sum) | O] of at most two parts to a run
extern "C" int64_t bf1_decode_fp8_workspace_bytes(int32_t batch, int32_t hq, int32_t hkv, int32_t max_degree, int32_t d) {
    if (batch < 0 || hq <= 0 || hkv <= 0 || hq % hkv != 0 || max_degree <= 0 || d <= 0) return -1;
    if (batch > kD8MaxScan) return 16;
    const size_t parts = (size_t)std::max(1, kD8MaxRuns / hkv) * hkv * 2 * (hq / hkv);
    return (int64_t)(up16(sizeof(int32_t) * ((size_t)batch + 2)) + parts * (sizeof(float2) + sizeof(float) * d));
}

// cu_tokens_dev null: `rows` is the batch.
static int decode8(const void* q, int32_t rows, const int32_t* cu_tokens_dev, const void* k_pages, const void* v_pages, const float* k_scales,
                   const float* v_scales, int32_t num_pages, const int32_t* seqlens_dev, int32_t batch, int32_t hq, int32_t hkv, int32_t d,
                   float softmax_scale, const bf1_decode_plan* plan, void* workspace, void* o, float* lse, void* stream) {
    if (!q || !k_pages || !v_pages || !k_scales || !v_scales || !seqlens_dev || !plan || !workspace || !o || !lse)
        return fail(BF1_ERR_INVALID_ARG, "a pointer is null");
    if (!plan->count || !plan->page || !plan->block || !plan->status) return fail(BF1_ERR_INVALID_ARG, "a decode-plan pointer is null");
    if (batch < 0 || rows < 0 || num_pages < 1 || hq <= 0 || hkv <= 0) return fail(BF1_ERR_INVALID_ARG, "negative or zero size argument");
    if (hq % hkv != 0) return fail(BF1_ERR_INVALID_ARG, "hq %d is not a multiple of hkv %d", hq, hkv);
    const int group = hq / hkv;
    if (group != 1 && group != 2 && group != 4) return fail(BF1_ERR_UNSUPPORTED, "GQA group size %d: only G = 1, 2 and 4 are supported", group);
    if (d != 64 && d != 128) return fail(BF1_ERR_UNSUPPORTED, "head dimension %d: only 64 and 128 are supported", d);
    if (((uintptr_t)q | (uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)o | (uintptr_t)workspace) & 15)
        return fail(BF1_ERR_INVALID_ARG, "q, k_pages, v_pages, o and workspace must be 16-byte aligned");
    if (plan->max_degree < 1 || batch > 65535 || hkv > 65535 || num_pages > (1 << 25) - 1 || (int64_t)plan->max_degree * std::min(batch, kD8MaxScan) > 0x7fffffffLL)
        return fail(BF1_ERR_UNSUPPORTED, "batch and KV heads up to 65535, pages up to 2^25 - 1, pages of all lists below 2^31");
    if (batch == 0 || rows == 0) return BF1_OK;
    Decode8Args a;
    a.q = (const __nv_bfloat16*)q;
    a.k_scales = k_scales;
    a.v_scales = v_scales;
    a.seqlens = seqlens_dev;
    a.count = plan->count;
    a.page = plan->page;
    a.block = plan->block;
    a.cu_tokens = cu_tokens_dev;
    a.status = plan->status;
    a.rows = rows;
    a.max_degree = plan->max_degree;
    a.hq = hq;
    a.hkv = hkv;
    a.num_pages = num_pages;
    a.group = group;
    a.batch = batch;
    a.scale_log2 = (softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)d)) * 1.4426950408889634f;
    a.o = (__nv_bfloat16*)o;
    a.lse = lse;
    int dev = 0;
    BF1_CUDA_CHECK(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return fail(BF1_ERR_NO_DEVICE, "device ordinal %d out of range", dev);
    static const Decode8Variant variants[4] = {decode8_variant<64, 2>(), decode8_variant<128, 2>(), decode8_variant<64, 4>(), decode8_variant<128, 4>()};
    const int heads = group == 4 ? 4 : 2, which = (group == 4 ? 2 : 0) + (d == 128), page_bytes = 2 * kP8 * d;
    const Decode8Variant& variant = variants[which];
    constexpr int kMostSmem = 144 * 1024;
    static std::atomic<int> sm_count[64];      // 0: this device has not been set up
    int sms = sm_count[dev].load(std::memory_order_acquire);
    if (!sms) {
        for (const Decode8Variant& v : variants)
            for (Decode8Kernel k : v.by_mode) {
                BF1_CUDA_CHECK(cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem));
                if (k == v.by_mode[kParts]) BF1_CUDA_CHECK(cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
            }
        BF1_CUDA_CHECK(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
        sm_count[dev].store(sms, std::memory_order_release);
    }
    const int64_t lists = (int64_t)batch * hkv;
    const int most = plan->max_degree;
    auto ceil_div = [](int64_t x, int64_t y) { return (int)((x + y - 1) / y); };
    // Which way, by what the host knows: the number of lists and the longest that there may be.  Over 784 shapes (1 to 1120 lists of up to 1
    // to 400 pages, d = 64 and 128, two and four heads; lists alike, from short to the longest evenly, and mostly short ones; on pages that no cache
    // holds) this takes 1.2 % longer on average than the best of the three.  us in runs / whole / in parts (16 query / 8 KV heads, d = 128):
    //   up to two pages a cluster never pays: one sequence of 1 / 2 pages 2.9 / 3.3 whole, 4.1 / 3.9 in parts;
    //   lists for every SM: 32 sequences of 12 pages 19.5 / 12.9 / 14.6, 140 of 4 27 / 25 / 26, 32 alike of 48 40 / 34 / 38, 64 of 48 71 / 87 / 83,
    //     64 of up to 48, mostly short, 26 / 39 / 30;
    //   fewer, in parts of up to 20 pages: one sequence of 12 / 48 / 200 / 400 pages 9.2 / 7.3 / 4.4, 11.7 / 23 / 7.5, 15.4 / 84 / 13.3, 19.7 / 164 / 20.0,
    //     eight of 48 / 200 18.6 / 23 / 14.3, 41 / 85 / 38, of up to 200, mostly short, 20.9 / 83 / 21.7.  Longer parts lose little where lists are alike and
    //     all where one is alone: 16000 tokens beside eleven sequences of 958 17 in runs, 29 in parts of 52 pages (4 KV heads).
    int mode = kRuns;
    if (batch > kD8MaxScan || most <= 2 || (lists >= sms && most <= 24)) mode = kWhole;
    else if (lists < sms && most <= 20 * kD8MaxCtas) mode = kParts;
    a.runs = a.nctas = a.share = 0;
    size_t smem = 1024;
    if (mode == kParts) {
        // as many CTAs to a list as still let all clusters run at once (a cluster's CTAs share a GPC, so this is less than what the SMs hold)
        for (int ctas = (int)std::min<int64_t>({kD8MaxCtas, most, (3 * (int64_t)sms + lists - 1) / lists}); mode == kParts; --ctas) {
            const int pages = ceil_div(most, ctas);      // of a CTA, at most
            if (pages > 20) mode = kRuns;
            ctas = ceil_div(most, pages);                // (no more than that takes)
            a.nctas = ctas;
            a.share = ceil_div(heads * d / 32, ctas) * 32;
            a.stages = std::min(pages, d == 128 ? 4 : 8);
            smem = 1024 + up16((size_t)ctas * heads * 8) + (size_t)ctas * a.share * 4;
            if (ctas == 1) break;
            int fit = 0;
            if (int rc = clusters8_that_fit(variant.by_mode[kParts], dev, which, ctas, a.stages, smem + (size_t)a.stages * page_bytes, &fit)) return rc;
            if (lists <= fit) break;
        }
    }
    if (mode == kRuns) {
        // three CTAs of three pages each to an SM: 24 lists of 32K tokens and less, all heads, 130 us; with two CTAs of four to six pages 134 to 137,
        // three of four 141 (more pages in flight than HBM needs wait for one another).  d = 64, where a CTA takes two pages at a step: 40 lists of 20000 tokens,
        // two heads, 42.6 us with six pages, 44.3 with four or eight, 44.1 with four CTAs, 45.8 page by page
        a.nctas = a.share = 0;
        smem = 1024 + sizeof(int) * (batch + 1);
        a.runs = std::max(1, std::min(3 * sms, kD8MaxRuns) / hkv);
        a.stages = d == 128 ? 3 : 6;
    } else if (mode == kWhole) {
        // Two CTAs to an SM with a ring of six pages, or, where there are more lists than that, three with four (d = 64: four): 320 / 384 / 512 / 1120 lists of 11 pages,
        // d = 128, 14.5 / 15.6 / 24.2 / 40.3 us, 22.1 / 23.6 / 25.4 / 48.4 with two CTAs in as many waves as that takes; 512 of 12, d = 64, 18.1 and 13.1
        a.stages = std::min(most, lists > 2 * sms ? (d == 128 ? 4 : 6) : (d == 128 ? 6 : 8));
    }
    // not the whole ring at the start: the first page would land later (32 sequences of 12 pages 12.4 us with all six at once, 12.2 with three)
    a.ahead = mode == kRuns ? 2 : 3;
    smem += (size_t)a.stages * page_bytes;
    a.bases = (int32_t*)workspace;
    a.part_ml = (float2*)((uint8_t*)workspace + up16(sizeof(int32_t) * ((size_t)batch + 2)));
    a.part_o = (float*)(a.part_ml + (size_t)hkv * a.runs * 2 * group);
    CUtensorMap tk, tv;
    if (int rc = make_page_map(&tk, k_pages, num_pages, hkv, d)) return rc;
    if (int rc = make_page_map(&tv, v_pages, num_pages, hkv, d)) return rc;
    const dim3 grid(hkv, mode == kRuns ? a.runs : batch, mode == kParts ? a.nctas : 1);
    BF1_CUDA_CHECK(launch_pdl_cluster(variant.by_mode[mode], grid, dim3(1, 1, grid.z), kD8Threads, smem, (cudaStream_t)stream, tk, tv, a));
    if (mode == kRuns)
        BF1_CUDA_CHECK(launch_pdl(d == 128 ? decode8_join_kernel<128> : decode8_join_kernel<64>, dim3(hkv, batch, std::max(1, group * d / 4 / kJoinColumns)),
                                  kJoinThreads, 0,
                                  (cudaStream_t)stream, a));
    return BF1_OK;
}

extern "C" int bf1_decode_fwd_fp8(const void* q, const void* k_pages, const void* v_pages, const float* k_scales, const float* v_scales,
                                  int32_t num_pages, const int32_t* seqlens_dev, int32_t batch, int32_t hq, int32_t hkv, int32_t d,
                                  float softmax_scale, const bf1_decode_plan* plan, void* workspace, void* o, float* lse, void* stream) {
    return decode8(q, batch, nullptr, k_pages, v_pages, k_scales, v_scales, num_pages, seqlens_dev, batch, hq, hkv, d, softmax_scale, plan, workspace, o, lse,
                   stream);
}

extern "C" int bf1_decode_fwd_fp8_packed(const void* q, int32_t tokens, const int32_t* cu_tokens_dev, const void* k_pages, const void* v_pages,
                                         const float* k_scales, const float* v_scales, int32_t num_pages, const int32_t* seqlens_dev, int32_t batch,
                                         int32_t hq, int32_t hkv, int32_t d, float softmax_scale, const bf1_decode_plan* plan, void* workspace, void* o,
                                         float* lse, void* stream) {
    if (!cu_tokens_dev) return fail(BF1_ERR_INVALID_ARG, "a pointer is null");
    return decode8(q, tokens, cu_tokens_dev, k_pages, v_pages, k_scales, v_scales, num_pages, seqlens_dev, batch, hq, hkv, d, softmax_scale, plan, workspace, o,
                   lse, stream);
}
