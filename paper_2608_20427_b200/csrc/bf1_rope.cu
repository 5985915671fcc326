// Rotary positions on the queries and keys of a packed batch, and on their gradients.
//
// A pair of dimensions (x, y) of a head at position p becomes (x cos a - y sin a, x sin a + y cos a) with a = p * f_i, the pair's
// frequency.  Every value is read once and written once, 4 bytes in all: bound by HBM for long batches, by one chain of launch,
// position, table and row for short ones.  The angles would be the arithmetic to pay for (64-bit product, sine and cosine); they are
// made once for a token and turn the same pairs of every head.  Measured (16 query / 8 KV heads, d = 128): 32768 tokens 64.3 us, 6.27 TB/s, 97 % of a
// copy; eight tokens 1.9 us in a graph.
#include <math.h>

#include <algorithm>

#include "bf1_rope.cuh"

namespace bf1 {

// Heads asked for before the first of them is turned: more CTAs on an SM count for more than more loads of each.  1 / 2 / 3 / 4 / 6: 4096
// tokens of 24 heads, forward and gradient, 22.7 / 19.8 / 23.1 / 23.5 / 23.0 us, 32768 forward 65.3 / 64.1 / 67.5 / 67.2 / 66.0.
constexpr int kRopeAhead = 2;
struct RopeArgs {
    Rows q, k, out_q, out_k;
    const int32_t* positions;
    RopeTable rope;
    int32_t tokens, hq, heads;     // heads: of q and k together
    float sign;
};

// blockIdx.x: tokens; blockIdx.y: one of gridDim.y shares of the heads
template <int D, int kSplit>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeArgs a) {
    constexpr int kWarps = kSplit > 1 ? 1 : 4;           // that share the heads
    pdl_wait();
    rope_block<D, kRopeAhead, kSplit>(a.rope, a.positions, (int64_t)blockIdx.x * kRopeTokens<D, kSplit>, a.tokens, a.sign, a.q, a.k, a.out_q, a.out_k,
                                      a.hq, a.heads, kWarps * blockIdx.y, kWarps * gridDim.y);
}

int check_rows(const bf1_rows* rows, const char* name) {
    if (!rows || !rows->data) return fail(BF1_ERR_INVALID_ARG, "%s is null", name);
    if (((uintptr_t)rows->data & 15) || rows->row_stride % 8 || rows->head_stride % 8)
        return fail(BF1_ERR_INVALID_ARG, "%s: its rows must be 16-byte aligned (strides in steps of 8 elements)", name);
    return BF1_OK;
}

int check_rope(const bf1_rope* rope, int32_t d) {
    if (!rope || !rope->turns) return fail(BF1_ERR_INVALID_ARG, "the rope or its table is null");
    if (rope->layout != BF1_ROPE_HALF && rope->layout != BF1_ROPE_INTERLEAVED)
        return fail(BF1_ERR_INVALID_ARG, "rope layout %d", rope->layout);
    if (rope->dim < 16 || rope->dim % 16 || rope->dim > d)
        return fail(BF1_ERR_UNSUPPORTED, "rotated dimensions %d: a multiple of 16 up to the head's %d", rope->dim, d);
    return BF1_OK;
}

static int rope_call(const bf1_rows* q, const bf1_rows* k, const int32_t* positions_dev, int32_t tokens, int32_t hq, int32_t hkv,
                     int32_t d, const bf1_rope* rope, const bf1_rows* out_q, const bf1_rows* out_k, float sign, void* stream) {
    if (tokens < 0 || hq < 1 || hkv < 0) return fail(BF1_ERR_INVALID_ARG, "bad token or head count");
    if (d != 64 && d != 128) return fail(BF1_ERR_UNSUPPORTED, "head dimension %d: only 64 and 128 are supported", d);
    if ((int64_t)hq + hkv > 65535) return fail(BF1_ERR_UNSUPPORTED, "%d query and %d KV heads", hq, hkv);
    if (tokens == 0) return BF1_OK;
    if (!positions_dev) return fail(BF1_ERR_INVALID_ARG, "positions is null");
    if (int rc = check_rope(rope, d)) return rc;
    const bf1_rows* rows[4] = {q, out_q, k, out_k};
    const char* const names[4] = {"q", "out_q", "k", "out_k"};
    for (int i = 0; i < (hkv ? 4 : 2); ++i)
        if (int rc = check_rows(rows[i], names[i])) return rc;
    for (int i = 0; i < (hkv ? 4 : 2); i += 2)
        if (rows[i]->data == rows[i + 1]->data && (rows[i]->row_stride != rows[i + 1]->row_stride || rows[i]->head_stride != rows[i + 1]->head_stride))
            return fail(BF1_ERR_INVALID_ARG, "%s in place of %s has to have its strides", names[i + 1], names[i]);
    RopeArgs a;
    a.q = rows_of(q);
    a.out_q = rows_of(out_q);
    a.k = hkv ? rows_of(k) : a.q;
    a.out_k = hkv ? rows_of(out_k) : a.out_q;
    a.positions = positions_dev;
    a.rope = table_of(rope);
    a.tokens = tokens;
    a.hq = hq;
    a.heads = hq + hkv;
    a.sign = sign;
    // Fewer than four heads: a warp for each would leave the others without (with the write of a cache behind it, 18000 tokens of one head 22 us, 16 with
    // tokens of its own for each warp).
    // Few tokens: their heads are shared out among CTAs.
    static void (*const kernels[2][2])(RopeArgs) = {{rope_kernel<64, 1>, rope_kernel<128, 1>}, {rope_kernel<64, 4>, rope_kernel<128, 4>}};
    const bool split = a.heads < 4;
    const int per_cta = (d == 128 ? kRopeTokens<128> : kRopeTokens<64>) * (split ? 4 : 1), ctas = (tokens + per_cta - 1) / per_cta;
    const int shares = split ? 1 : std::max(1, std::min((a.heads + 3) / 4, 148 * 8 / ctas));
    BF1_CUDA_CHECK(launch_pdl(kernels[split][d == 128], dim3(ctas, shares), kRopeThreads, 0, (cudaStream_t)stream, a));
    return BF1_OK;
}

}  // namespace bf1

using namespace bf1;

extern "C" int bf1_rope_turns(const bf1_rope_cfg* cfg, double* turns, double* magnitude) {
    if (!cfg || !turns || !magnitude) return fail(BF1_ERR_INVALID_ARG, "a pointer is null");
    if (cfg->dim < 16 || cfg->dim % 16) return fail(BF1_ERR_UNSUPPORTED, "rotated dimensions %d: a multiple of 16", cfg->dim);
    if (!(cfg->base > 1.0) || !isfinite(cfg->base)) return fail(BF1_ERR_INVALID_ARG, "the base has to be above 1");
    const bool scaled = cfg->scaling != BF1_ROPE_NONE;
    if (scaled && cfg->scaling != BF1_ROPE_LINEAR && cfg->scaling != BF1_ROPE_NTK && cfg->scaling != BF1_ROPE_YARN)
        return fail(BF1_ERR_INVALID_ARG, "rope scaling %d", cfg->scaling);
    if (scaled && (!(cfg->factor >= 1.0) || !isfinite(cfg->factor)))
        return fail(BF1_ERR_INVALID_ARG, "the factor of a scaled rope has to be 1 or more");
    if (cfg->scaling == BF1_ROPE_YARN && !(cfg->original_len >= 1.0 && cfg->beta_fast > cfg->beta_slow && cfg->beta_slow >= 0.0 &&
                                           isfinite(cfg->original_len) && isfinite(cfg->beta_fast)))
        return fail(BF1_ERR_INVALID_ARG, "yarn wants original_len >= 1 and beta_fast > beta_slow >= 0");
    const double r = cfg->dim;
    const double base = cfg->scaling == BF1_ROPE_NTK ? cfg->base * pow(cfg->factor, r / (r - 2.0)) : cfg->base;
    for (int i = 0; i < cfg->dim / 2; ++i) {
        double t = pow(base, -2.0 * i / r) / (2.0 * 3.14159265358979323846);
        if (cfg->scaling == BF1_ROPE_LINEAR) t /= cfg->factor;
        if (cfg->scaling == BF1_ROPE_YARN) {
            double keep = (cfg->original_len * t - cfg->beta_slow) / (cfg->beta_fast - cfg->beta_slow);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            t = keep * t + (1.0 - keep) * t / cfg->factor;
        }
        turns[i] = t;
    }
    *magnitude = cfg->scaling == BF1_ROPE_YARN ? 0.1 * log(cfg->factor) + 1.0 : 1.0;
    return BF1_OK;
}

extern "C" int bf1_rope_fwd(const bf1_rows* q, const bf1_rows* k, const int32_t* positions_dev, int32_t tokens, int32_t hq, int32_t hkv,
                            int32_t d, const bf1_rope* rope, const bf1_rows* out_q, const bf1_rows* out_k, void* stream) {
    return rope_call(q, k, positions_dev, tokens, hq, hkv, d, rope, out_q, out_k, 1.f, stream);
}

extern "C" int bf1_rope_bwd(const bf1_rows* d_q, const bf1_rows* d_k, const int32_t* positions_dev, int32_t tokens, int32_t hq, int32_t hkv,
                            int32_t d, const bf1_rope* rope, const bf1_rows* out_q, const bf1_rows* out_k, void* stream) {
    return rope_call(d_q, d_k, positions_dev, tokens, hq, hkv, d, rope, out_q, out_k, -1.f, stream);
}
