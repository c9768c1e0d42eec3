// C entry points of the orthogonalised update: the plan (sizes, tables, tensor maps) and its two calls.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <functional>
#include <memory>

#include "api_util.h"
#include "ortho.h"

using namespace gvq;
using namespace gvq::ortho;

struct gvq_ortho {
    gvq_ctx *ctx = nullptr;
    int device = 0;              // (destroying the plan does not touch the context, which may be gone)
    Device dev{};
    SmallPlan small{};           // where all matrices fit an SM or a cluster of them
    void *tables = nullptr;      // one device allocation: matrices, tensor maps, tiles, chunks, partial sums
};

namespace {

constexpr size_t kAlign = 256;
// A part of a contraction: at least so many stages, at most so many parts.  Against (6, 4), time with (6, 8), (12, 4), (9, 3):
// 515 x 1027 +0, +2, +2 %; twice 512 x 4608 +0, +0, -8 %; the VGG-16-shaped weights +0, +0, +2 %.
constexpr int kPartStages = 6, kMaxParts = 4;
constexpr int kTileCost = 3;      // what a tile costs beyond its contraction, in stages of 64 steps
// Pairs of CTAs on 256 x 256 tiles from this many multiply-adds of one X P on, 128 x 64 tiles below.  Measured on either side,
// us per step of bf16 weights in pairs / alone: 1500 x 1500 (3.4e9) 284 / 217, four 512 x 4608 (4.8e9) 262 / 272, 1700 x 1700
// (4.9e9) 306 / 287, five 1024 x 1024 (5.4e9) 307 / 265, 1850 x 1850 (6.3e9) 277 / 282, six 1024 x 1024 (6.4e9) 317 / 290,
// six 512 x 4608 (7.2e9) 337 / 354, eight 1024 x 1024 (8.6e9) 316 / 350, 2048 x 2048 (8.6e9) 288 / 326.
constexpr int64_t kPairWork = 6'800'000'000;
size_t up(size_t n) { return (n + kAlign - 1) & ~(kAlign - 1); }
int up32(int n) { return (n + 31) & ~31; }     // rows of the work arrays: whole pieces of 32 entries

struct Sizes {
    std::vector<Matrix> mats;
    size_t bytes = 0;            // of the workspace
};

// The matrices of a layout and the workspace they take, laid out from `base` (null: sizes only).
gvq_status lay_out(int n_layers, const int64_t *off, const int64_t *len, const int32_t *rows, const int32_t *cols,
                   const float *scales, unsigned char *base, Sizes &out)
{
    for (int l = 0; l < n_layers; ++l) {
        if (rows[l] == 0 && cols[l] == 0) continue;               // not a matrix: left alone
        if (rows[l] < 1 || cols[l] < 1 || (int64_t)rows[l] * cols[l] != len[l]) return GVQ_ERR_SHAPE;
        if (rows[l] > INT32_MAX - 512 || cols[l] > INT32_MAX - 512) return GVQ_ERR_SHAPE;
        Matrix m{};
        m.rows = rows[l]; m.cols = cols[l];
        m.r = std::min(m.rows, m.cols); m.c = std::max(m.rows, m.cols);
        if (m.r > 32768 || m.c >= 1 << 20) return GVQ_ERR_SHAPE;  // beyond any layer
        m.tall = m.rows > m.cols;
        m.ldx = up32(m.cols); m.ldr = up32(m.r);
        m.off = off[l];
        m.by_cols = ((uint64_t)1 << 62) / (uint64_t)m.cols + 1;
        // entries of X have an rms of 1 / sqrt(r c) at first and 1 / sqrt(c) at last: about 1 / sqrt(r) to 1 when scaled
        m.sx = std::exp2(std::round(0.5f * std::log2((float)m.c)));
        m.scale = scales ? scales[l] : std::sqrt(std::max(1.0f, (float)m.rows / (float)m.cols));
        auto take = [&](size_t entries) {
            __half *p = reinterpret_cast<__half *>(base ? base + out.bytes : nullptr);
            out.bytes += up(entries * sizeof(__half));
            return p;
        };
        const size_t nx = (size_t)m.rows * m.ldx, nr = (size_t)m.r * m.ldr;
        m.x[0] = take(nx); m.x[1] = take(nx); m.lo = take(nx); m.gram = take(nr); m.poly = take(nr);
        m.split = m.r <= kSplitApply ? 2 : m.r <= kSplitSide ? 1 : 0;
        if (m.split > 0) m.gram_lo = take(nr);
        if (m.split > 1) m.poly_lo = take(nr);
        out.mats.push_back(m);
    }
    return GVQ_OK;
}

bool encode(EncodeTiledFn enc, CUtensorMap *map, void *p, int rows, int cols, int ld, int box_rows)
{
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld * sizeof(__half)};
    cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, p, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Deals tiles to at most `units` CTAs so that their costs come out even (longest first, to whoever has least), and puts
// each one's tiles together, a matrix's next to each other.  Returns where the runs start.
std::vector<int32_t> deal(std::vector<Tile> &tiles, int units)
{
    auto cost = [&](const Tile &t) { return t.k1 - t.k0 + kTileCost; };
    std::stable_sort(tiles.begin(), tiles.end(), [&](const Tile &a, const Tile &b) { return cost(a) > cost(b); });
    const int runs = (int)std::min<size_t>(units, tiles.size());
    std::vector<std::vector<Tile>> run(runs);
    std::vector<std::pair<int64_t, int>> heap;       // (load, run), least on top
    for (int i = 0; i < runs; ++i) heap.push_back({0, i});
    const auto more = std::greater<std::pair<int64_t, int>>();
    for (const Tile &t : tiles) {
        std::pop_heap(heap.begin(), heap.end(), more);
        run[heap.back().second].push_back(t);
        heap.back().first += cost(t);
        std::push_heap(heap.begin(), heap.end(), more);
    }
    std::vector<int32_t> start{0};
    tiles.clear();
    for (auto &r : run) {
        tiles.insert(tiles.end(), r.begin(), r.end());
        start.push_back((int32_t)tiles.size());
    }
    return start;
}

// Cuts contractions that are longer than a CTA's share of all of them.  `pieces`: of 32 x 64 entries in a tile.
void split(std::vector<Tile> &tiles, int units, int pieces, int &slots)
{
    int64_t total = 0;
    for (const Tile &t : tiles) total += t.k1;
    const int64_t share = std::max<int64_t>(kPartStages, (total + units - 1) / units);
    std::vector<Tile> out;
    for (const Tile &t : tiles) {
        const int parts = (int)std::min<int64_t>(kMaxParts, (t.k1 + share - 1) / share);
        for (int i = 0; i < parts; ++i) {
            Tile s = t;
            s.k0 = (int)((int64_t)t.k1 * i / parts);
            s.k1 = (int)((int64_t)t.k1 * (i + 1) / parts);
            s.part = i;
            s.parts = parts;
            s.slot = slots;
            out.push_back(s);
        }
        if (parts > 1) slots += parts * pieces;
    }
    tiles = out;
}

// The whole update: one launch where every matrix fits an SM or a cluster of them, otherwise two element-wise ones and three a step.
gvq_status run(gvq_ortho *p, const ElementArgs &in, const OutputArgs &out)
{
    gvq_ctx *ctx = p->ctx;
    DeviceGuard guard(ctx->device);
    if (p->small.room > 0) {
        GVQ_CUDA(ctx, launch_small(ctx->stream, p->dev.mats, p->dev.n_mats, p->small, in, out, ctx->error_word,
                                   ctx->wait_kcycles, ctx->drop_last_load));
        return GVQ_OK;
    }
    GVQ_CUDA(ctx, launch_start(ctx->stream, p->dev, in));
    for (int s = 0; s < kSteps; ++s)
        for (Phase ph : {kGram, kPoly, kApply})
            GVQ_CUDA(ctx, launch_product(ctx->stream, p->dev, ph, s, &out, ctx->error_word, ctx->wait_kcycles, ctx->drop_last_load));
    return GVQ_OK;
}

bool finite(float x) { return std::isfinite(x); }

}  // namespace

extern "C" {

int64_t gvq_ortho_workspace_bytes(const gvq_layout *layout, const int32_t *rows, const int32_t *cols)
{
    if (!rows || !cols || gvq_layout_check(layout) != GVQ_OK) return -1;
    try {
        Sizes s;
        if (lay_out(layout->n_layers, layout->layer_off, layout->layer_len, rows, cols, nullptr, nullptr, s) != GVQ_OK) return -1;
        return (int64_t)s.bytes;
    } catch (const std::exception &) {       // no host memory
        return -1;
    }
}

gvq_status gvq_ortho_create(gvq_ortho **out, gvq_ctx *ctx, const int32_t *rows, const int32_t *cols, const float *scales_opt,
                            void *workspace, size_t workspace_bytes)
{
    if (!out) return GVQ_ERR_NULL;
    *out = nullptr;
    if (!ctx || !rows || !cols) return GVQ_ERR_NULL;
    if (!ctx->encode_fn) return GVQ_ERR_UNSUPPORTED;
    try {
        Sizes sz;
        gvq_status st = lay_out(ctx->n_layers, ctx->layer_off.data(), ctx->layer_len.data(), rows, cols, scales_opt,
                                static_cast<unsigned char *>(workspace), sz);
        if (st != GVQ_OK) return st;
        if (scales_opt)
            for (int l = 0; l < ctx->n_layers; ++l)
                if (!finite(scales_opt[l])) return GVQ_ERR_SHAPE;
        if (sz.bytes > 0 && (!workspace || workspace_bytes < sz.bytes)) return GVQ_ERR_WORKSPACE;
        if ((reinterpret_cast<uintptr_t>(workspace) & (kAlign - 1)) != 0) return GVQ_ERR_ALIGN;

        const int n = (int)sz.mats.size();
        std::vector<CUtensorMap> maps((size_t)n * kMaps);
        std::vector<Tile> sym, apply;
        std::vector<Chunk> chunks;
        int64_t entries = 0;
        for (const Matrix &m : sz.mats) entries += (int64_t)m.rows * m.cols;
        const int chunk = (int)std::min<int64_t>(kMaxChunk, std::max<int64_t>(kMinChunk, entries / (4 * ctx->num_sms) / kMinChunk * kMinChunk));
        for (int i = 0; i < n; ++i) {
            Matrix &m = sz.mats[i];
            CUtensorMap *mp = &maps[(size_t)i * kMaps];
            auto map = [&](int which, __half *p, int box_rows, bool square) {
                return encode((EncodeTiledFn)ctx->encode_fn, mp + which, p, square ? m.r : m.rows, square ? m.r : m.cols,
                              square ? m.ldr : m.ldx, box_rows);
            };
            if (!map(kX0, m.x[0], 64, false) || !map(kX1, m.x[1], 64, false) || !map(kGramMap, m.gram, 64, true) ||
                !map(kPolyMap, m.poly, 64, true) || !map(kX0Out, m.x[0], 32, false) || !map(kX1Out, m.x[1], 32, false) ||
                !map(kLoOut, m.lo, 32, false) || !map(kGramOut, m.gram, 32, true) || !map(kPolyOut, m.poly, 32, true))
                return GVQ_ERR_CUDA;
            if (m.split > 0 && (!map(kGramLoMap, m.gram_lo, 64, true) || !map(kGramLoOut, m.gram_lo, 32, true))) return GVQ_ERR_CUDA;
            if (m.split > 1 && (!map(kPolyLoMap, m.poly_lo, 64, true) || !map(kPolyLoOut, m.poly_lo, 32, true))) return GVQ_ERR_CUDA;
            m.chunk0 = (int)chunks.size();
            m.n_chunks = (int)(((int64_t)m.rows * m.cols + chunk - 1) / chunk);
            for (int k = 0; k < m.n_chunks; ++k) chunks.push_back({i, k});
        }
        std::vector<Tile> gram;
        int64_t apply_work = 0;
        for (const Matrix &m : sz.mats) apply_work += (int64_t)m.r * m.r * m.c;
        const bool pair = apply_work >= kPairWork;
        {
            const int64_t bm = pair ? 256 : 128, bn = pair ? kPairN : kSoloN;
            for (int i = 0; i < n; ++i) {
                const Matrix &m = sz.mats[i];
                const int kr = (m.r + 63) / 64, kc = (m.c + 63) / 64;
                const int poly_terms = m.split > 0 ? 3 : 1, apply_terms = m.split > 1 ? 2 : 1;     // products of halves
                // tiles of a symmetric product: those that reach the diagonal or lie right of it
                for (int tm = 0; tm * bm < m.r; ++tm)
                    for (int tn = (int)(tm * bm / bn); tn * bn < m.r; ++tn) {
                        gram.push_back({i, tm, tn, 0, kc, 0, 1, 0});
                        sym.push_back({i, tm, tn, 0, poly_terms * kr, 0, 1, 0});
                    }
                for (int tm = 0; tm * bm < m.rows; ++tm)
                    for (int tn = 0; tn * bn < m.cols; ++tn) apply.push_back({i, tm, tn, 0, apply_terms * kr, 0, 1, 0});
            }
        }
        const int units = pair ? ctx->num_sms / 2 : ctx->num_sms;
        int slots = 0;
        split(gram, units, (pair ? 2 : 1) * 4 * (pair ? kPairN : kSoloN) / 64, slots);
        const std::vector<int32_t> gram_start = deal(gram, units), sym_start = deal(sym, units), apply_start = deal(apply, units);

        std::unique_ptr<gvq_ortho> p(new gvq_ortho());
        p->ctx = ctx;
        p->device = ctx->device;
        std::vector<unsigned char> image;
        auto put = [&](const void *src, size_t bytes) {
            const size_t at = up(image.size());
            image.resize(at + bytes);
            if (bytes) std::memcpy(image.data() + at, src, bytes);
            return at;
        };
        auto table = [&](const auto &v) { return put(v.data(), sizeof(v[0]) * v.size()); };
        const size_t o_m = table(sz.mats), o_t = table(maps), o_g = table(gram), o_s = table(sym), o_a = table(apply), o_c = table(chunks),
                     o_gs = table(gram_start), o_ss = table(sym_start), o_as = table(apply_start);
        const std::vector<int32_t> no_tickets((size_t)slots, 0);
        const size_t o_k = table(no_tickets);
        // behind the image: sums of squares, and the parts' sums
        const size_t o_p = up(image.size()), o_q = o_p + up(sizeof(float) * chunks.size()), all = o_q + (size_t)slots * 8192;
        DeviceGuard guard(ctx->device);
        cudaError_t e = cudaMalloc(&p->tables, all + kAlign);
        if (e == cudaSuccess) e = upload(p->tables, image.data(), image.size());
        if (e != cudaSuccess) {
            if (p->tables) cudaFree(p->tables);
            return cuda_fail(ctx, e);
        }
        unsigned char *t = static_cast<unsigned char *>(p->tables);
        Device &d = p->dev;
        d.mats = reinterpret_cast<Matrix *>(t + o_m);
        d.maps = reinterpret_cast<CUtensorMap *>(t + o_t);
        auto work = [&](Run &r, size_t tiles, size_t start, const std::vector<int32_t> &s) {
            r.tiles = reinterpret_cast<Tile *>(t + tiles);
            r.start = reinterpret_cast<int32_t *>(t + start);
            r.runs = (int)s.size() - 1;
        };
        work(d.run[kGram], o_g, o_gs, gram_start);
        work(d.run[kPoly], o_s, o_ss, sym_start);
        work(d.run[kApply], o_a, o_as, apply_start);
        d.run[kLast] = d.run[kApply];
        d.chunks = reinterpret_cast<Chunk *>(t + o_c);
        d.n_chunks = (int)chunks.size();
        d.tickets = reinterpret_cast<int32_t *>(t + o_k);
        d.n_tickets = slots;
        d.partial = reinterpret_cast<float *>(t + o_p);
        d.parts = reinterpret_cast<float *>(t + o_q);
        d.pair = pair;
        for (const Matrix &m : sz.mats) d.split = std::max(d.split, m.split);
        d.n_mats = n;
        int shorter = 0, longer = 0;
        for (const Matrix &m : sz.mats) {
            shorter = std::max(shorter, m.r);
            longer = std::max(longer, m.c);
        }
        p->small = small_plan(n, shorter, longer, ctx->num_sms);
        d.chunk = chunk;
        *out = p.release();
        return GVQ_OK;
    } catch (const std::exception &) {       // no host memory
        return GVQ_ERR_CUDA;
    }
}

gvq_status gvq_ortho_destroy(gvq_ortho *p)
{
    if (!p) return GVQ_OK;
    DeviceGuard guard(p->device);
    if (p->tables) cudaFree(p->tables);
    delete p;
    return GVQ_OK;
}

gvq_status gvq_orthogonalize(gvq_ortho *p, const float *g, void *out, int dtype)
{
    if (!p || !g || !out) return GVQ_ERR_NULL;
    if (dtype != GVQ_F32 && dtype != GVQ_BF16 && dtype != GVQ_F16) return GVQ_ERR_SHAPE;
    if (static_cast<const void *>(g) == out) return GVQ_ERR_SHAPE;
    if (!aligned16(g) || !aligned16(out)) return GVQ_ERR_ALIGN;
    if (p->dev.n_chunks == 0) return GVQ_OK;
    return run(p, {g, nullptr, 0.0f, 0}, {out, dtype, 0, 0.0f, 0.0f});
}

gvq_status gvq_ortho_step(gvq_ortho *p, const float *g, float *momentum, float beta, int nesterov, void *w, int dtype, float lr,
                          float weight_decay)
{
    if (!p || !g || !momentum || !w) return GVQ_ERR_NULL;
    if (dtype != GVQ_F32 && dtype != GVQ_BF16 && dtype != GVQ_F16) return GVQ_ERR_SHAPE;
    if (!(beta >= 0.0f && beta < 1.0f) || !finite(lr) || !finite(weight_decay)) return GVQ_ERR_SHAPE;
    if (g == momentum || static_cast<const void *>(g) == w || static_cast<void *>(momentum) == w) return GVQ_ERR_SHAPE;
    if (!aligned16(g) || !aligned16(momentum) || !aligned16(w)) return GVQ_ERR_ALIGN;
    if (p->dev.n_chunks == 0) return GVQ_OK;
    return run(p, {g, momentum, beta, nesterov}, {w, dtype, 1, 1.0f - lr * weight_decay, lr});
}

}  // extern "C"
