// Host side of the orthogonalised update: validation, workspace planning, the products of every phase, launches.
//
// The iteration X <- a X + (b A + c A^2) X, A = X X^T, is a sequence of products that depend on one another; the
// matrices of a list do not.  So a list is worked on in groups, one launch for all products of a group, whose tiles
// are listed product by product: the first product of every matrix, the second of every matrix, and so on.
// Two ways to take steps, P = a I + B:
//   one by one   A = X X^T, B = b A + c A^2, X <- P X
//   two together A, B as before, T = P A, A' = P T (= X' X'^T of the step in between, without X'),
//                B' = b A' + c A'^2, Q = P' P, X <- Q X
// The second form replaces two long products (m x n) by three m x m ones: taken from n = 1.5 m on, where it also has fewer
// tile k-blocks, from m = 256 on, and for the first two steps only.  There it costs no accuracy: what A' loses beside X' X'^T
// is what rounding X' would have lost.  Later steps would lose more: an error of A' is absolute, while a direction that the
// input holds little of has grown to a few hundredths by then and counts with its square (nearly square matrices have many).
// How many there are depends on the input, not on its shape: rows or columns of different size make a wide matrix act like a
// nearly square one.
// (64-bit models of the code's arithmetic, bfloat16, five steps, error of X: one by one, 2 + 1 + 1 + 1, 2 + 2 + 1, 3 + 1 + 1, 3 + 2.
//   2048 x 5461, normal                                 0.93e-3  0.87e-3  1.20e-3  0.87e-3  0.82e-3
//   the same, columns scaled by 10^-1 ... 10            1.08e-3  1.01e-3  1.31e-3  1.08e-3  2.19e-3
//   the same, 10^-2 ... 10^2                            1.05e-3  0.98e-3  1.47e-3  1.08e-3  3.14e-3
//   384 x 256, normal                                   1.05e-3  1.06e-3  1.41e-3  1.55e-3  1.54e-3
//   384 x 256, rows scaled by 10^-2 ... 10^2            1.20e-3  1.19e-3  3.62e-3  1.91e-3  3.76e-3
//   64 x 1000, heavy tails, worst of six                1.45e-3  2.29e-3
// the last is why m = 256: fewer directions average less.  The kernels bear the model out to 5 %; fp32 weights, 5461 x 2048,
// rows scaled by 10^-1 ... 10: 3.2e-5 as 2 + 1 + 1 + 1, 1.1e-4 as 3 + 2.  Orthogonalising a 7B layer takes 12.0 ms, 11.1 as 3 + 1 + 1,
// 10.2 as 3 + 2.)
// A, B, T, A', B', Q are polynomials of one symmetric matrix: symmetric, so only half their tiles are computed.
//
// Rounding.  What is stored in 16 bits has 11 of them, and how much of the identity B + s I holds matters:
//   16-bit floats     s = a: the products that use P read nothing beside their operands, and nothing is added in their
//                     epilogues.  64-bit models of this arithmetic on normal gradients (512 x 512 ... 1024 x 2736): X is
//                     1.0e-3 ... 1.3e-3 off; the rounding of the bfloat16 result is 1.65e-3.  (s such that B + s I lies near 0 where most singular values are near 1, and
//                     (a - s) X added in fp32: 0.8e-3 ... 1.0e-3, and 15 % more time for a 60M model's 28 matrices, 2 % for
//                     a 7B layer: not done.)
//   pairs             the second form: the sums of the tensor cores lose more on a X + B X as one product than the
//                     fp32 addition does (200 x 200, five steps: 6e-6 instead of 2e-6).
#include "../../include/apollo.h"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "apollo_internal.h"
#include "muon.h"

using namespace apollo;

namespace {

constexpr size_t ALIGN = 256;
constexpr int MAX_SIDE = 1 << 20;
constexpr int S_BUFS = 3;                                 // m x m matrices at a time
constexpr int TOGETHER_FROM = 256;                        // short side
constexpr int64_t WIDE_FROM = 660, SMALL_UP_TO = 800;     // k-blocks, see make_plan

size_t align_up(size_t x) { return (x + ALIGN - 1) / ALIGN * ALIGN; }
int round_up(int x, int to) { return (x + to - 1) / to * to; }

struct Mat {
    int rows, cols, m, n, tall, pitch_x, pitch_s, n_part;
    bool together;                       // the first two steps
    size_t x[2][2], s[S_BUFS][2], part;  // workspace offsets: [buffer][high, low]
    size_t maps;                         // offset of its tensor maps
};

struct Group {
    std::vector<int> mats;
    int tile;                            // which of MUON_TILES
    int64_t tile_begin, tiles;           // in the list of tiles
};

// The powers of two that stored values carry, and the constants of the iteration.
struct Scales { double x, a, b, t, q, shift, q_shift; };     // B + shift I, Q - q_shift I are stored

struct Plan {
    std::vector<Mat> mats;
    std::vector<Group> groups;
    size_t off_status, off_counters, off_table, table_bytes, off_maps, off_ops, off_list, total;
    int n_ops, maps_per_mat, parts;
    int64_t n_tiles;
    Scales sc;
};

// Whether iterates are sums of two 16-bit floats.
bool split_of(const apollo_muon_config& cfg) { return cfg.dtype == APOLLO_DT_F32 || cfg.products == APOLLO_MUON_PRODUCTS_PAIRS; }

double poly(const float* c, double x) { const double y = x * x; return x * (c[0] + y * (c[1] + y * c[2])); }

// Bounds of everything stored, from the iteration on [0, 1] (the singular values of X start there).
bool find_scales(const apollo_muon_config& cfg, Scales& sc)
{
    const double a = cfg.coef[0], b = cfg.coef[1], c = cfg.coef[2];
    const int N = 8192;
    double top = 1.0, now = 1.0;
    for (int k = 0; k < cfg.ns_steps; ++k) {
        double next = 0.0;
        for (int i = 0; i <= N; ++i) next = std::max(next, std::fabs(poly(cfg.coef, now * i / N)));
        now = next;
        if (!(now <= 8.0)) return false;
        top = std::max(top, now);
    }
    double b_min = 0.0, b_max = 0.0, t_max = 0.0, p_max = 0.0;
    for (int i = 0; i <= N; ++i) {
        const double y = top * top * i / N, v = y * (b + c * y), p = a + v;
        b_min = std::min(b_min, v); b_max = std::max(b_max, v);
        t_max = std::max(t_max, std::fabs(y * p));
        p_max = std::max(p_max, std::fabs(p));
    }
    const bool fold = !split_of(cfg);
    sc.shift = fold ? a : -(0.7 * b_min + 0.3 * b_max);
    sc.q_shift = fold ? 0.0 : 1.0;
    // the largest power of two that keeps a value of this size at or below 2^15 (16-bit floats end at 65504)
    auto scale_for = [](double v) { return std::exp2(std::floor(15.0 - std::log2(std::max(v, 1.0)))); };
    sc.x = scale_for(top);
    sc.a = scale_for(top * top);
    sc.b = scale_for(std::max(b_max - b_min, 1.0) + std::fabs(sc.shift));
    sc.t = scale_for(t_max);
    sc.q = scale_for(p_max * p_max + sc.q_shift);
    return true;
}

int validate(const apollo_muon_config* cfg, Scales& sc)
{
    if (!cfg) return APOLLO_ERR_INVALID_ARG;
    if (cfg->dtype != APOLLO_DT_F32 && cfg->dtype != APOLLO_DT_BF16) return APOLLO_ERR_INVALID_ARG;
    if (cfg->ns_steps < 1 || cfg->ns_steps > APOLLO_MUON_MAX_STEPS) return APOLLO_ERR_INVALID_ARG;
    for (float c : cfg->coef)
        if (!std::isfinite(c)) return APOLLO_ERR_INVALID_ARG;
    if (!(cfg->momentum >= 0.0f && cfg->momentum < 1.0f) || (cfg->nesterov != 0 && cfg->nesterov != 1)) return APOLLO_ERR_INVALID_ARG;
    if (cfg->scale < APOLLO_MUON_SCALE_NONE || cfg->scale > APOLLO_MUON_SCALE_RMS) return APOLLO_ERR_INVALID_ARG;
    if (!std::isfinite(cfg->eps) || !(cfg->eps > 0.0f)) return APOLLO_ERR_INVALID_ARG;
    if (cfg->products != APOLLO_MUON_PRODUCTS_DEFAULT && cfg->products != APOLLO_MUON_PRODUCTS_PAIRS) return APOLLO_ERR_INVALID_ARG;
    if (cfg->workspace_mb < 0 || cfg->workspace_mb > 65536) return APOLLO_ERR_INVALID_ARG;
    return find_scales(*cfg, sc) ? APOLLO_OK : APOLLO_ERR_INVALID_ARG;
}

int tiles_of(int x, int per) { return (x + per - 1) / per; }

// Tiles of a symmetric m x m product: blocks of a tile's rows against the columns from the block's own on.
int64_t sym_tiles(int m, const MuonTile& tile)
{
    int64_t t = 0;
    for (int tm = 0; tm < tiles_of(m, tile.m); ++tm) t += tiles_of(m, tile.n) - (int64_t)tm * (tile.m / tile.n);
    return t;
}
int64_t full_tiles(int m, int n, const MuonTile& tile) { return (int64_t)tiles_of(m, tile.m) * tiles_of(n, tile.n); }

// Steps that the update at step k takes.
int joint(bool together, int steps, int k) { return together && k == 0 ? std::min(2, steps) : 1; }
int updates_of(bool together, int steps)
{
    int n = 0;
    for (int k = 0; k < steps; k += joint(together, steps, k)) ++n;
    return n;
}

// Products of a matrix: an update by j steps has A and X, j times B, j - 1 times T, A' and Q.
int products_of(bool together, int steps) { return 4 * steps - updates_of(together, steps); }

// Tile k-blocks of all products: what a pair of CTAs works off.
double cost(int m, int n, bool together, int steps)
{
    const double km = tiles_of(m, 64), kn = tiles_of(n, 64), sym = (double)sym_tiles(m, MUON_TILES[TILE_WIDE]);
    const double up = (double)full_tiles(m, n, MUON_TILES[TILE_WIDE]) * km;
    const int updates = updates_of(together, steps);
    return updates * (sym * kn + up) + (products_of(together, steps) - 2 * updates) * sym * km;
}

int64_t all_tiles(const Mat& m, int steps, const MuonTile& tile)
{
    const int up = updates_of(m.together, steps);
    return up * full_tiles(m.m, m.n, tile) + (products_of(m.together, steps) - up) * sym_tiles(m.m, tile);
}

int make_plan(const apollo_shape* shapes, int32_t n_mat, const apollo_muon_config* cfg, Plan& plan)
{
    if (!shapes || n_mat < 1) return APOLLO_ERR_INVALID_ARG;
    const int rc = validate(cfg, plan.sc);
    if (rc != APOLLO_OK) return rc;
    plan.parts = split_of(*cfg) ? 2 : 1;
    plan.maps_per_mat = (2 + S_BUFS) * MUON_MAPS * plan.parts;
    plan.mats.resize(n_mat);
    std::vector<size_t> need(n_mat);
    for (int i = 0; i < n_mat; ++i) {
        const int64_t rows = shapes[i].rows, cols = shapes[i].cols;
        if (rows < 1 || cols < 1 || rows > MAX_SIDE || cols > MAX_SIDE) return APOLLO_ERR_SHAPE;
        Mat& m = plan.mats[i];
        m.rows = (int)rows; m.cols = (int)cols;
        m.tall = rows > cols;
        m.m = m.tall ? m.cols : m.rows;
        m.n = m.tall ? m.rows : m.cols;
        m.pitch_x = round_up(m.n, 64);
        m.pitch_s = round_up(m.m, 64);
        const int64_t numel = rows * cols;
        m.n_part = (int)std::min<int64_t>(MUON_PART, (numel + 8191) / 8192);
        m.together = m.m >= TOGETHER_FROM && 2 * m.n >= 3 * m.m && cost(m.m, m.n, true, cfg->ns_steps) < cost(m.m, m.n, false, cfg->ns_steps);
        size_t off = 0;
        for (int b = 0; b < 2; ++b)
            for (int h = 0; h < plan.parts; ++h) { m.x[b][h] = off; off = align_up(off + 2 * (size_t)m.m * m.pitch_x); }
        for (int b = 0; b < S_BUFS; ++b)
            for (int h = 0; h < plan.parts; ++h) { m.s[b][h] = off; off = align_up(off + 2 * (size_t)m.m * m.pitch_s); }
        m.part = off; off = align_up(off + sizeof(double) * (size_t)m.n_part);
        need[i] = off;
    }
    // groups: like matrices together (their phases then end together), as many as fit
    std::vector<int> order(n_mat);
    for (int i = 0; i < n_mat; ++i) order[i] = i;
    std::stable_sort(order.begin(), order.end(), [&](int p, int q) {
        const Mat &x = plan.mats[p], &y = plan.mats[q];
        if (x.m != y.m) return x.m > y.m;
        return x.n > y.n;
    });
    const size_t budget = (size_t)(cfg->workspace_mb ? cfg->workspace_mb : 2048) << 20;
    plan.groups.clear();
    size_t used = 0, largest = 0;
    for (int i : order) {
        if (plan.groups.empty() || (used > 0 && used + need[i] > budget)) { plan.groups.push_back(Group()); used = 0; }
        Mat& m = plan.mats[i];
        for (auto& b : m.x) for (size_t& o : b) o += used;
        for (auto& b : m.s) for (size_t& o : b) o += used;
        m.part += used;
        used += need[i];
        largest = std::max(largest, used);
        plan.groups.back().mats.push_back(i);
    }
    plan.n_ops = 0; plan.n_tiles = 0;
    for (Group& g : plan.groups) {
        // Wide tiles move the fewest bytes per product; the others shorten a product (its tiles are loaded and stored by
        // more CTAs), which is what counts as long as there are few.  By the k-blocks of one m x m product of all matrices,
        // five steps of apollo_muon_orthogonalize in us, wide tiles against 256 x 128:  288 (12 of 512 x 512) 146, 123;  480 (20 of
        // 512 x 512) 155, 145;  640 (four of 1024 x 1024) 188, 179;  672 (28 of 512 x 512) 173, 169;  672 (a 60M model's 28, eight of
        // them 512 x 1376, four 1376 x 512) 230, 239;  800 (five of 1024) 197, 198;  1152 (one 2048) 270, 297.
        // The same count in tiles of 128 x 128, these against 256 x 128:  80 (one 512 x 512) 94, 108;  576 (one 1024) 137,
        // 151;  640 (eight of 512) 109, 116;  960 (twelve of 512) 125, 123;  1100 (one 1280) 189, 174;  1872 (one 1536) 294, 199.
        // (fp32, three times the k-blocks, changes sides at the same counts: 480: 365, 321;  640: 459, 429;  1152: 701, 762;  and
        // 576: 309, 354;  640: 226, 243;  960: 279, 262.  Long sides, which the counts leave out, change them earlier: two
        // of 1024 x 4096, 320: 276, 283;  one of them, 576 small: 278, 252.)
        int64_t wide = 0, small = 0;
        for (int i : g.mats) {
            const int m = plan.mats[i].m;
            wide += sym_tiles(m, MUON_TILES[TILE_WIDE]) * tiles_of(m, 64);
            small += sym_tiles(m, MUON_TILES[TILE_SMALL]) * tiles_of(m, 64);
        }
        g.tile = wide >= WIDE_FROM ? TILE_WIDE : small <= SMALL_UP_TO ? TILE_SMALL : TILE_TALL;
        g.tile_begin = plan.n_tiles;
        g.tiles = 0;
        for (int i : g.mats) {
            g.tiles += all_tiles(plan.mats[i], cfg->ns_steps, MUON_TILES[g.tile]);
            plan.n_ops += products_of(plan.mats[i].together, cfg->ns_steps);
        }
        if (g.tiles > INT32_MAX / 2) return APOLLO_ERR_SHAPE;
        plan.n_tiles += g.tiles;
    }
    if (plan.n_ops > 1 << TILE_OP_BITS) return APOLLO_ERR_SHAPE;
    static_assert(MAX_SIDE / 128 <= 1 << TILE_M_BITS && MAX_SIDE / 128 <= 1 << TILE_N_BITS && 3 * (MAX_SIDE / 64) < 1 << TILE_K_BITS,
                  "the fields of a tile hold the longest sides, three segments of the contraction included");
    size_t off = 0;
    plan.off_status = off; off += ALIGN;
    plan.off_counters = off; off = align_up(off + sizeof(uint32_t) * ((size_t)n_mat + 1));   // the ticket, then one per matrix
    plan.off_table = off;
    plan.off_maps = off; off = align_up(off + 128 * (size_t)plan.maps_per_mat * n_mat);
    plan.off_ops = off; off = align_up(off + sizeof(GemmOp) * (size_t)plan.n_ops);
    plan.off_list = off; off = align_up(off + sizeof(uint64_t) * (size_t)plan.n_tiles);
    plan.table_bytes = off - plan.off_table;
    for (int i = 0; i < n_mat; ++i) {
        Mat& m = plan.mats[i];
        for (auto& b : m.x) for (size_t& o : b) o += off;
        for (auto& b : m.s) for (size_t& o : b) o += off;
        m.part += off;
        m.maps = plan.off_maps + 128 * (size_t)plan.maps_per_mat * i;
    }
    plan.total = off + largest;
    return APOLLO_OK;
}

}  // namespace

struct apollo_muon_ctx {
    apollo_muon_config cfg;
    Plan plan;
    char* ws;
    char* table;          // pinned host copy of the device tables
    bool pinned;
    bool first;
    int last_launches;
    MuonLaunch launch;
};

namespace {

// The products of one matrix, in order.
void ops_of(const apollo_muon_ctx* ctx, int index, const MuonTile& tile, std::vector<GemmOp>& out)
{
    const Mat& m = ctx->plan.mats[index];
    const Plan& plan = ctx->plan;
    const Scales& sc = plan.sc;
    const double a = ctx->cfg.coef[0], b = ctx->cfg.coef[1], c = ctx->cfg.coef[2], p = a - sc.shift;
    const int parts = plan.parts;
    char* ws = ctx->ws;
    auto x_map = [&](int buf, int h, int kind) { return (const void*)(ws + m.maps + 128 * (size_t)((buf * parts + h) * MUON_MAPS + kind)); };
    auto s_map = [&](int buf, int h, int kind) { return x_map(2 + buf, h, kind); };
    auto x_ptr = [&](int buf, int h) { return (const __half*)(ws + m.x[buf][h]); };
    auto s_ptr = [&](int buf, int h) { return (const __half*)(ws + m.s[buf][h]); };
    // the loads of L, and of R with k contiguous: a CTA's half of the tile, 128 or 64 rows
    const int l_kind = tile.m == 256 ? MAP_ROWS : MAP_COLS, r_kind = tile.n == 256 ? MAP_ROWS : MAP_COLS;
    uint32_t* counter = reinterpret_cast<uint32_t*>(ws + plan.off_counters) + 1 + index;
    uint32_t done = 0;
    auto push = [&](GemmOp& o) {
        o.counter = counter;
        o.need = done;
        done += MUON_COUNTS_PER_TILE * (uint32_t)(o.sym ? sym_tiles(o.M, tile) : full_tiles(o.M, o.N, tile));
        out.push_back(o);
    };
    auto square = [&](int l, int r, int dst, double alpha, int e1, double b1, int e2, double b2, double diag, bool of_x) {
        GemmOp o;
        std::memset(&o, 0, sizeof(o));
        for (int h = 0; h < parts; ++h) {
            o.l_map[h] = of_x ? x_map(l, h, l_kind) : s_map(l, h, l_kind);
            o.r_map[h] = of_x ? x_map(r, h, r_kind) : s_map(r, h, r_kind);
            o.out_map[h] = s_map(dst, h, MAP_STORE);
            o.mir_map[h] = s_map(dst, h, MAP_MIRROR);
            if (b1 != 0.0) o.e1[h] = s_ptr(e1, h);
            if (b2 != 0.0) o.e2[h] = s_ptr(e2, h);
        }
        o.alpha = (float)alpha; o.b1 = (float)b1; o.b2 = (float)b2; o.diag = (float)diag;
        o.M = o.N = m.m; o.K = of_x ? m.n : m.m; o.e_pitch = m.pitch_s;
        o.sym = 1;
        push(o);
    };
    auto update = [&](int s, int src, double alpha, double b1) {
        GemmOp o;
        std::memset(&o, 0, sizeof(o));
        for (int h = 0; h < parts; ++h) {
            o.l_map[h] = s_map(s, h, l_kind);
            o.r_map[h] = x_map(src, h, MAP_COLS);
            o.out_map[h] = x_map(src ^ 1, h, MAP_STORE);
            if (b1 != 0.0) o.e1[h] = x_ptr(src, h);
        }
        o.alpha = (float)alpha; o.b1 = (float)b1;
        o.M = m.m; o.N = m.n; o.K = m.m; o.e_pitch = m.pitch_x;
        o.r_mn = 1;
        push(o);
    };
    // polynomials of one matrix commute, so these products of two of them are symmetric too
    auto poly_b = [&](int s, int dst) { square(s, s, dst, c * sc.b / (sc.a * sc.a), 0, b * sc.b / sc.a, -1, 0, sc.shift * sc.b, false); };
    int x = 0;
    for (int k = 0; k < ctx->cfg.ns_steps; x ^= 1) {
        const int steps = joint(m.together, ctx->cfg.ns_steps, k);
        k += steps;
        square(x, x, 0, sc.a / (sc.x * sc.x), -1, 0, -1, 0, 0, true);                                   // S0 = A
        poly_b(0, 1);                                                                                   // S1 = B + s I
        if (steps == 1) { update(1, x, 1.0 / sc.b, p); continue; }
        square(1, 0, 2, sc.t / (sc.b * sc.a), 0, p * sc.t / sc.a, -1, 0, 0, false);                     // S2 = T = P A
        square(1, 2, 0, sc.a / (sc.b * sc.t), 2, p * sc.a / sc.t, -1, 0, 0, false);                     // S0 = A' = P T
        poly_b(0, 2);                                                                                   // S2 = B' + s I
        square(2, 1, 0, sc.q / (sc.b * sc.b), 1, p * sc.q / sc.b, 2, p * sc.q / sc.b, (p * p - sc.q_shift) * sc.q, false);      // S0 = Q = P' P - q I
        update(0, x, 1.0 / sc.q, sc.q_shift);
    }
}

// Fills the host copy of the tables.
int build_table(apollo_muon_ctx* ctx)
{
    Plan& plan = ctx->plan;
    char* t = ctx->table;                                   // corresponds to ws + off_table
    auto at = [&](size_t off) { return t + (off - plan.off_table); };
    for (size_t i = 0; i < plan.mats.size(); ++i) {
        const Mat& m = plan.mats[i];
        char* maps = at(m.maps);
        for (int b = 0; b < 2 + S_BUFS; ++b)
            for (int h = 0; h < plan.parts; ++h, maps += 128 * MUON_MAPS) {
                const size_t at_ws = b < 2 ? m.x[b][h] : m.s[b - 2][h];
                const int rc = muon_encode_maps((const __half*)(ctx->ws + at_ws), m.m, b < 2 ? m.n : m.m, b < 2 ? m.pitch_x : m.pitch_s, maps);
                if (rc != APOLLO_OK) return rc;
            }
    }
    GemmOp* d_ops = reinterpret_cast<GemmOp*>(at(plan.off_ops));
    uint64_t* list = reinterpret_cast<uint64_t*>(at(plan.off_list));
    int op = 0;
    for (const Group& g : plan.groups) {
        std::vector<std::vector<GemmOp>> ops(g.mats.size());
        size_t products = 0;
        for (size_t k = 0; k < g.mats.size(); ++k) {
            ops_of(ctx, g.mats[k], MUON_TILES[g.tile], ops[k]);
            products = std::max(products, ops[k].size());
        }
        uint64_t* out = list + g.tile_begin;
        for (size_t p = 0; p < products; ++p)
            for (size_t k = 0; k < g.mats.size(); ++k) {
                if (p >= ops[k].size()) continue;
                const GemmOp& o = ops[k][p];
                d_ops[op] = o;
                const MuonTile& tile = MUON_TILES[g.tile];
                const int rows = tiles_of(o.M, tile.m), cols = tiles_of(o.N, tile.n), per = tile.m / tile.n;
                const uint32_t kb = (uint32_t)(plan.parts == 2 ? 3 : 1) * (uint32_t)tiles_of(o.K, 64);
                // column by column: the tiles at work at one time share few columns of R and all rows of L
                for (int tn = 0; tn < cols; ++tn)
                    for (int tm = 0; tm < (o.sym ? std::min(rows, tn / per + 1) : rows); ++tm)
                        *out++ = pack_tile((uint32_t)op, (uint32_t)tm, (uint32_t)tn, kb, (uint32_t)o.r_mn);
                ++op;
            }
        if (out != list + g.tile_begin + g.tiles) return APOLLO_ERR_INVALID_ARG;      // the plan counted otherwise
    }
    return APOLLO_OK;
}

double gain_of(const apollo_muon_config& cfg, const Mat& m)
{
    if (cfg.scale == APOLLO_MUON_SCALE_SHAPE) return std::sqrt(std::max(1.0, (double)m.rows / m.cols));
    if (cfg.scale == APOLLO_MUON_SCALE_RMS) return 0.2 * std::sqrt((double)std::max(m.rows, m.cols));
    return 1.0;
}

// `step`: momentum and weights; else U in d_G, O in d_W.
int run(apollo_muon_ctx* ctx, void* const* d_W, const void* const* d_G, float* const* d_M, float lr, float wd, bool step, void* cuda_stream)
{
    if (!ctx || !d_W || !d_G || (step && !d_M)) return APOLLO_ERR_INVALID_ARG;
    if (!std::isfinite(lr) || !std::isfinite(wd)) return APOLLO_ERR_INVALID_ARG;
    const Plan& plan = ctx->plan;
    for (size_t i = 0; i < plan.mats.size(); ++i) {
        if (!d_W[i] || !d_G[i] || (step && !d_M[i])) return APOLLO_ERR_INVALID_ARG;
        if ((uintptr_t)d_W[i] % 16 || (uintptr_t)d_G[i] % 16 || (step && (uintptr_t)d_M[i] % 16)) return APOLLO_ERR_ALIGN;
    }
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int32_t* d_status = reinterpret_cast<int32_t*>(ctx->ws + plan.off_status);
    if (ctx->first) {
        // A capture would only record the upload: the tables would be missing until the graph is launched.
        cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
        if (cudaStreamIsCapturing(stream, &capture) != cudaSuccess || capture != cudaStreamCaptureStatusNone) {
            cudaGetLastError();
            return APOLLO_ERR_INVALID_ARG;
        }
        if (cudaMemsetAsync(d_status, 0, ALIGN, stream) != cudaSuccess ||
            cudaMemcpyAsync(ctx->ws + plan.off_table, ctx->table, plan.table_bytes, cudaMemcpyHostToDevice, stream) != cudaSuccess) {
            cudaGetLastError();
            return APOLLO_ERR_CUDA;
        }
    }
    const GemmOp* d_ops = reinterpret_cast<const GemmOp*>(ctx->ws + plan.off_ops);
    const uint64_t* d_list = reinterpret_cast<const uint64_t*>(ctx->ws + plan.off_list);
    uint32_t* d_ticket = reinterpret_cast<uint32_t*>(ctx->ws + plan.off_counters);
    const int dtype = ctx->cfg.dtype;
    const bool split = plan.parts == 2;
    int launches = 0;
    cudaError_t err = cudaSuccess;
    for (const Group& g : plan.groups) {
        // streaming passes: up to MUON_CHUNK matrices a launch, their pointers as kernel parameters
        auto pass = [&](int which) {
            for (size_t at = 0; at < g.mats.size() && err == cudaSuccess; at += MUON_CHUNK) {
                MuonArgs a;
                a.n = (int)std::min<size_t>(MUON_CHUNK, g.mats.size() - at);
                a.mu = ctx->cfg.momentum; a.eps = ctx->cfg.eps; a.x_scale = (float)plan.sc.x; a.lr = lr; a.wd = wd; a.nesterov = ctx->cfg.nesterov;
                a.ticket = d_ticket;
                int64_t tiles = 0;
                for (int k = 0; k < a.n; ++k) {
                    const int i = g.mats[at + k];
                    const Mat& m = plan.mats[i];
                    MuonItem& it = a.item[k];
                    const int buf = which == 2 ? updates_of(m.together, ctx->cfg.ns_steps) & 1 : 0;
                    it.w = d_W[i]; it.g = d_G[i]; it.m = step ? d_M[i] : nullptr;
                    it.x[0] = reinterpret_cast<__half*>(ctx->ws + m.x[buf][0]);
                    it.x[1] = plan.parts == 2 ? reinterpret_cast<__half*>(ctx->ws + m.x[buf][1]) : nullptr;
                    it.part = reinterpret_cast<double*>(ctx->ws + m.part);
                    it.counter = d_ticket + 1 + i;
                    it.rows = m.rows; it.cols = m.cols; it.x_pitch = m.pitch_x; it.n_part = m.n_part; it.tall = m.tall;
                    it.gain = (float)gain_of(ctx->cfg, m);
                    a.tile_begin[k] = (int)tiles;
                    tiles += which == 0 ? m.n_part : muon_stream_tiles(m.rows, m.cols, m.tall != 0, which == 2);
                }
                for (int k = a.n; k <= MUON_CHUNK; ++k) a.tile_begin[k] = (int)tiles;
                if (tiles > INT32_MAX) { err = cudaErrorInvalidValue; return; }
                if (which == 0) err = launch_muon_moment(dtype, step, a, (int)tiles, d_status, stream);
                else if (which == 1) err = launch_muon_load(dtype, split, step, a, (int)tiles, d_status, stream);
                else err = launch_muon_apply(dtype, split, step, a, (int)tiles, d_status, stream);
                ++launches;
            }
        };
        pass(0);
        pass(1);
        if (err == cudaSuccess) {
            err = launch_muon_gemm(split, g.tile, d_ops, d_list + g.tile_begin, (int)g.tiles, d_ticket, ctx->launch, d_status, stream);
            ++launches;
        }
        pass(2);
    }
    if (err != cudaSuccess) { cudaGetLastError(); return APOLLO_ERR_CUDA; }
    ctx->first = false;
    ctx->last_launches = launches;
    return APOLLO_OK;
}

}  // namespace

extern "C" {

int apollo_muon_workspace_bytes(const apollo_shape* shapes, int32_t n_matrices, const apollo_muon_config* cfg, size_t* out_bytes)
{
    if (!out_bytes) return APOLLO_ERR_INVALID_ARG;
    try {
        Plan plan;
        const int rc = make_plan(shapes, n_matrices, cfg, plan);
        if (rc != APOLLO_OK) return rc;
        *out_bytes = plan.total;
        return APOLLO_OK;
    } catch (...) {
        return APOLLO_ERR_INVALID_ARG;
    }
}

int apollo_muon_create(apollo_muon_ctx** out_ctx, const apollo_shape* shapes, int32_t n_matrices, const apollo_muon_config* cfg,
                       void* d_workspace, size_t workspace_bytes)
{
    if (!out_ctx) return APOLLO_ERR_INVALID_ARG;
    *out_ctx = nullptr;
    apollo_muon_ctx* ctx = new (std::nothrow) apollo_muon_ctx();
    if (!ctx) return APOLLO_ERR_INVALID_ARG;
    ctx->table = nullptr;
    ctx->pinned = false;
    int rc;
    try {
        rc = make_plan(shapes, n_matrices, cfg, ctx->plan);
        if (rc == APOLLO_OK && !d_workspace) rc = APOLLO_ERR_INVALID_ARG;
        if (rc == APOLLO_OK && ((uintptr_t)d_workspace % ALIGN || workspace_bytes < ctx->plan.total)) rc = APOLLO_ERR_WORKSPACE;
        int device = 0, major = 0, sms = 0;
        if (rc == APOLLO_OK && (cudaGetDevice(&device) != cudaSuccess ||
                                cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, device) != cudaSuccess ||
                                cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess)) {
            cudaGetLastError();
            rc = APOLLO_ERR_CUDA;
        }
        if (rc == APOLLO_OK && major != 10) rc = APOLLO_ERR_UNSUPPORTED;
        if (rc == APOLLO_OK) {
            ctx->cfg = *cfg;
            ctx->ws = static_cast<char*>(d_workspace);
            ctx->first = true;
            ctx->last_launches = 0;
            ctx->launch = MuonLaunch{ sms, { 0, 0 } };
            void* host = nullptr;
            if (cudaHostAlloc(&host, ctx->plan.table_bytes, cudaHostAllocDefault) == cudaSuccess) {
                ctx->pinned = true;
            } else {
                cudaGetLastError();                     // no pinned memory to be had: the upload goes from pageable memory
                host = new char[ctx->plan.table_bytes];
            }
            ctx->table = static_cast<char*>(host);
            std::memset(ctx->table, 0, ctx->plan.table_bytes);
            rc = build_table(ctx);
        }
    } catch (...) {
        rc = APOLLO_ERR_INVALID_ARG;
    }
    if (rc != APOLLO_OK) {
        apollo_muon_destroy(ctx);
        return rc;
    }
    *out_ctx = ctx;
    return APOLLO_OK;
}

int apollo_muon_destroy(apollo_muon_ctx* ctx)
{
    if (!ctx) return APOLLO_ERR_INVALID_ARG;
    if (ctx->table) {
        if (ctx->pinned) cudaFreeHost(ctx->table);      // waits for an upload in flight
        else delete[] ctx->table;
    }
    delete ctx;
    return APOLLO_OK;
}

int apollo_muon_step(apollo_muon_ctx* ctx, void* const* d_W, const void* const* d_G, float* const* d_M, float lr, float wd, void* cuda_stream)
{
    return run(ctx, d_W, d_G, d_M, lr, wd, true, cuda_stream);
}

int apollo_muon_orthogonalize(apollo_muon_ctx* ctx, const void* const* d_U, void* const* d_O, void* cuda_stream)
{
    return run(ctx, d_O, d_U, nullptr, 0.0f, 0.0f, false, cuda_stream);
}

int apollo_muon_status(apollo_muon_ctx* ctx, void* cuda_stream)
{
    if (!ctx) return APOLLO_ERR_INVALID_ARG;
    if (cudaStreamSynchronize(static_cast<cudaStream_t>(cuda_stream)) != cudaSuccess) return APOLLO_ERR_CUDA;
    if (ctx->first) return APOLLO_OK;                   // nothing has run; the status word is not initialised yet
    int32_t word = 0;
    char* d_status = ctx->ws + ctx->plan.off_status;
    if (cudaMemcpy(&word, d_status, sizeof(word), cudaMemcpyDeviceToHost) != cudaSuccess) return APOLLO_ERR_CUDA;
    if (word != STATUS_OK) {
        cudaMemset(d_status, 0, 2 * sizeof(word));
        return word == STATUS_BOUNDS ? APOLLO_ERR_INTERNAL : APOLLO_ERR_TIMEOUT;
    }
    return APOLLO_OK;
}

int apollo_muon_last_launches(const apollo_muon_ctx* ctx, int32_t* out)
{
    if (!ctx || !out) return APOLLO_ERR_INVALID_ARG;
    *out = ctx->last_launches;
    return APOLLO_OK;
}

}  // extern "C"
