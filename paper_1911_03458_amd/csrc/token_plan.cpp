// Plans and entry points of the operators along a sequence of tokens (include/merit_tokens.h): what is accepted, how a
// pass is split into workgroups, how much scratch memory it takes.  Host code only.
#include "token_plan.h"

using namespace merit;

namespace {

// ---- group norm ------------------------------------------------------------------------
// Column tiles and row chunks for `vec` channels a lane; returns the floats of scratch memory.
int64_t norm_layout(NormParams &p, int vec, bool backward)
{
    p.vec = vec;
    p.slab = 0;
    const int cu = p.Cg / vec;
    p.rows_form = p.S == 1 && cu <= 1024;
    if (p.rows_form) {
        const bool whole = cu > 256;                    // a workgroup has a row of the group
        int lg = 1;
        while (lg < 64 && lg < cu) lg *= 2;
        p.ctiles = whole ? p.G : (int)cdiv(p.G, 64 / lg);
        // eight wavefronts a SIMD; backward fewer: each leaves a row of sums behind
        const int64_t rows = whole ? p.N : cdiv(p.N, 4), most = cdiv(backward ? 1024 : 2048, p.ctiles);
        p.chunks = rows < most ? rows : most;
        p.chunk_rows = 1;
        return backward ? p.chunks * 2 * p.C : 0;
    }
    // A workgroup a group, where its registers hold the group's values (bfloat16, us a call, chunks / this: forward 1x196x512, 32
    // groups 9.6 / 5.7, 4x3136x256 12.1 / 8.9, 2 groups of 1x784x64 8.9 / 5.8; backward with 32 groups and more 15.9 / 9.8 and
    // 20.1 / 17.4, with 16 17.1 / 19.6, with 2 14.5 / 19.2).  Fewer than 128 units would leave most of its threads without one.
    // Not where rows of one unit each make many long groups (binary16, 8x3136x256 15.4 / 12.6, but 10 images 16.7 / 17.7, 32
    // 32.0 / 41.3; 16x1568x256 15.0 / 12.4, 32 20.4 / 22.9; 64x784x512 32.2 / 28.9): the line that such a row is a piece of comes
    // once for each group of it.  And not backward where eight channels a lane make many sums to leave (binary16, 8x49x2048 16.1 /
    // 15.4, but 16 16.5 / 17.8, 64 23.4 / 38.7; 16x196x1024 19.7 / 18.3, 64 34.1 / 39.9; fp32 64x196x1024 47.5 / 38.3).
    const bool torn = cu == 1 && p.S > 1024 && p.N * p.G * p.S > 900000;
    const bool sums = !backward || (p.N * p.G >= 32 && (vec < 8 || p.N * p.C <= 24576));
    if (vec > 1 && sums && !torn && cu <= 256 && p.S * cu >= 128) {
        for (int form : {0x104, 0x108, 0x404, 0x408}) {
            const int threads = form & 0x400 ? 1024 : 256, units = form & 0xFF;
            if (p.S > (int64_t)(threads / cu) * units || p.N * p.G * threads >= MAX_THREADS) continue;
            p.slab = form;
            p.ctiles = p.G;
            p.chunks = 1;
            p.chunk_rows = p.S;
            return backward ? p.N * 2 * p.C : 0;
        }
    }
    // Chunks: tiles of about 32 units side by side (512 bytes of a row), and so many row chunks that there are 1024 workgroups;
    // not more than eight for each thread that joins them in the second launch.
    const int pieces = (int)cdiv(cu, 256), fit = cu < 32 ? 32 / cu : 1, gt = pieces > 1 ? 1 : fit < p.G ? fit : p.G;
    p.group_tile = gt;
    p.ctiles = pieces > 1 ? p.G * pieces : (int)cdiv(p.G, gt);
    const int rw = pieces > 1 ? 1 : 256 / (gt * cu);
    int lanes = 64;
    while (lanes * gt > 256) lanes /= 2;
    int64_t chunks = cdiv(1024, p.ctiles * (p.N > 0 ? p.N : 1));
    const int64_t most = cdiv(p.S, 4 * rw);
    if (chunks > most) chunks = most;
    if (chunks > 8 * lanes) chunks = 8 * lanes;
    if (chunks < 1) chunks = 1;
    p.chunk_rows = cdiv(cdiv(p.S, chunks), rw) * rw;
    if (p.chunk_rows < 1) p.chunk_rows = 1;
    p.chunks = p.S > 0 ? cdiv(p.S, p.chunk_rows) : 1;
    const int64_t groups = p.N * p.G * p.chunks * pieces * 2;
    return groups + (backward ? p.N * p.chunks * 2 * p.C : p.N * p.G);
}
// channels a lane moves at once: the most of 16 bytes, 8, ... that divides a group, and that the rows' boundaries allow
template <typename F> int norm_vec(const NormParams &p, int type, F &&aligned)
{
    for (int vec = 16 / elem_bytes(type); vec > 1; vec /= 2)
        if (p.Cg % vec == 0 && aligned(vec)) return vec;
    return 1;
}
int64_t norm_bytes(const NormParams &p, int type, bool backward)
{
    int64_t most = 0;
    for (int vec = 16 / elem_bytes(type); vec >= 1; vec /= 2) {
        if (p.Cg % vec) continue;
        NormParams q = p;
        const int64_t n = norm_layout(q, vec, backward);
        if (n > most) most = n;
    }
    return most * 4;
}

// ---- causal convolution ---------------------------------------------------------------------
// Channels a lane moves at once, whatever their type: with eight of 16 bits a lane's window, taps and sums take so many registers
// that too few wavefronts are left to wait for memory (8x2048x2048 bfloat16, forward 36 us with 8, 29 with 4).
constexpr int CONV_VEC = 4;
// Tokens of a strip (it reads K - 1 rows again): the longest of 8, 16, 32 that gives every SIMD four wavefronts; backward of 8 to
// 64 that gives it two (bfloat16, forward 3x4099x1536: 16 tokens 16.8 us, 32 18.8, 64 27; backward 8x2048x2048: 16 60 us, 32 54,
// 64 50, 128 69).
int64_t conv_layout(CconvParams &p, int vec, bool backward)
{
    p.vec = vec;
    const int64_t cu = p.D / vec;
    p.strip = backward ? 64 : 32;
    while (p.strip > 8 && p.B * cdiv(p.L, p.strip) * cu < (backward ? 2 : 4) * 65536) p.strip /= 2;
    p.strips = p.L > 0 ? cdiv(p.L, p.strip) : 1;
    int ct = 1;
    while (ct < 64 && ct < cu) ct *= 2;
    p.row_blocks = cdiv(p.B * p.strips, 256 / ct);
    return backward ? p.row_blocks * (p.K + 1) * (int64_t)p.D : 0;
}
int64_t conv_blocks(const CconvParams &p)
{
    const int64_t cu = p.D / p.vec;
    int ct = 1;
    while (ct < 64 && ct < cu) ct *= 2;
    return p.row_blocks * cdiv(cu, ct);
}
int64_t conv_bytes(const CconvParams &p, int type, bool backward)
{
    CconvParams q = p;
    const int vec = CONV_VEC;
    int64_t most = conv_layout(q, 1, backward);
    if (p.D % vec == 0) {
        const int64_t n = conv_layout(q, vec, backward);
        if (n > most) most = n;
    }
    return most * 4;
}

// ---- scan ----------------------------------------------------------------------------------------
int64_t scan_part_bc(const ScanParams &p) { return (int64_t)p.G * p.ctiles * p.B * p.L * 2 * p.N; }
int64_t scan_part_a(const ScanParams &p) { return p.B * p.chunks * ((int64_t)p.D * p.N + 2 * p.D); }
int64_t scan_chunk_floats(const ScanParams &p) { return p.chunks > 1 ? p.B * p.chunks * (int64_t)p.D * (p.N + 1) : 0; }
// A sequence's chunks can run side by side, for a launch more that finds the state before each (the state that a chunk adds:
// most of a forward pass's arithmetic, a tenth of a backward one's) and a chunk's way through what those before it left.  What
// `chunks` cost, in hundredths of the time of a tile: 512 workgroups run at once, two a compute unit, and up to 256 of them
// take half of that time (8 states) or a little more.
int64_t scan_cost(const ScanParams &p, int64_t blocks, int64_t chunk_tiles, int64_t chunks, bool backward)
{
    const int64_t w = blocks * chunks, rest = w % 512;
    const int64_t half = p.N <= 8 ? 50 : backward && p.N <= 16 ? 60 : 55;
    const int64_t runs = chunk_tiles * (w / 512 * 100 + (rest == 0 ? 0 : rest <= 256 ? half : 100));
    if (chunks == 1) return runs;
    return backward ? runs + runs / 10 + 5 * chunks + 100 : runs + runs * 4 / 5 + 25 * chunks + 400;
}
// The cheapest of 1 to 4 sqrt(tiles) chunks of two tiles and more (bfloat16, D 2048, 16 states, us in one piece / in chunks /
// those: forward 1x8191 553 / 122 / 16, 1x512 39 / 17 / 8, 3x2048 141 / 93 / 8, 4x2048 142 / 119 / 4, but 6x2048 144 / 171 / 8;
// backward 1x8191 2753 / 327 / 16, 6x2048 713 / 473 / 8, 8x2048 720 / 595 / 2, but 16x1024 508 / 568 / 2).
void scan_layout(ScanParams &p, bool backward)
{
    const int cpb = SCAN_THREADS / scan_lpc(p.N);
    p.ctiles = (int)cdiv(p.Dg, cpb);
    p.tiles = cdiv(p.L, MERIT_SCAN_TILE);
    p.chunks = 1;
    p.chunk_tiles = p.tiles > 0 ? p.tiles : 1;
    const int64_t blocks = p.B * p.G * p.ctiles;
    if (blocks == 0 || blocks > 1024 || p.tiles < 4) return;
    int64_t most = cdiv(2048, blocks);
    if (most > p.tiles / 2) most = p.tiles / 2;
    while (most * most > 16 * p.tiles) --most;
    int64_t least = scan_cost(p, blocks, p.tiles, 1, backward);
    for (int64_t k = 2; k <= most; ++k) {
        const int64_t tiles = cdiv(p.tiles, k), chunks = cdiv(p.tiles, tiles), cost = scan_cost(p, blocks, tiles, chunks, backward);
        if (cost >= least) continue;
        least = cost;
        p.chunk_tiles = tiles;
        p.chunks = (int)chunks;
    }
}

}  // namespace

extern "C" {

merit_status merit_plan_group_norm(merit_dtype type, int64_t N, int64_t S, int64_t C, int64_t groups, double eps,
                                   merit_act act, merit_token_plan **out)
{
    if (!out) return MERIT_ERR_NULL;
    *out = nullptr;
    if (!type_ok(type) || (int)act < 0 || (int)act > 2 || N < 0 || S < 0 || C < 1 || groups < 1 || !(eps >= 0.0) ||
        !std::isfinite(eps))
        return MERIT_ERR_INVALID_ARG;
    if (C % groups != 0) return MERIT_ERR_SHAPE;
    if (C > MAX_CHANNELS || N > MAX_ROWS || S > MAX_ROWS || too_large(N, S, C)) return MERIT_ERR_UNSUPPORTED;
    merit_token_plan *pl = new_plan(NORM, type);
    if (!pl) return MERIT_ERR_INVALID_ARG;
    NormParams &p = pl->norm;
    p.N = N; p.S = S;
    p.C = (int)C; p.G = (int)groups; p.Cg = (int)(C / groups);
    p.eps = (float)eps;
    p.act = act;
    for (int vec = 16 / elem_bytes(type); vec >= 1; vec /= 2) {
        if (p.Cg % vec) continue;
        NormParams q = p;
        norm_layout(q, vec, true);              // (the pass with more workgroups of the two)
        const bool too_many = q.rows_form ? q.chunks * q.ctiles >= MAX_BLOCKS : q.N > MAX_BLOCKS || q.N * q.chunks * q.ctiles >= MAX_BLOCKS;
        norm_layout(q, vec, false);
        if (too_many || (q.rows_form ? q.chunks * q.ctiles >= MAX_BLOCKS : q.N > MAX_BLOCKS || q.N * q.chunks * q.ctiles >= MAX_BLOCKS)) {
            delete pl;
            return MERIT_ERR_UNSUPPORTED;
        }
    }
    *out = pl;
    return MERIT_OK;
}

merit_status merit_plan_causal_conv(merit_dtype type, int64_t B, int64_t L, int64_t D, int64_t K, merit_act act,
                                    merit_token_plan **out)
{
    if (!out) return MERIT_ERR_NULL;
    *out = nullptr;
    if (!type_ok(type) || (int)act < 0 || (int)act > 2 || B < 0 || L < 0 || D < 1 || K < 1) return MERIT_ERR_INVALID_ARG;
    if (K > MERIT_CONV_MAX_TAPS || D > MAX_CHANNELS || B > MAX_ROWS || L > MAX_ROWS || too_large(B, L, D))
        return MERIT_ERR_UNSUPPORTED;
    merit_token_plan *pl = new_plan(CONV, type);
    if (!pl) return MERIT_ERR_INVALID_ARG;
    CconvParams &p = pl->conv;
    p.B = B; p.L = L; p.D = (int)D; p.K = (int)K;
    p.act = act;
    for (int vec : {1, CONV_VEC}) {
        if (p.D % vec) continue;
        CconvParams q = p;
        conv_layout(q, vec, false);
        const int64_t more = cdiv(B * D * K, 256);             // single tokens, the first rows' gradient
        if (q.row_blocks >= MAX_BLOCKS || conv_blocks(q) >= MAX_BLOCKS || B > MAX_BLOCKS || more >= MAX_BLOCKS) {
            delete pl;
            return MERIT_ERR_UNSUPPORTED;
        }
    }
    *out = pl;
    return MERIT_OK;
}

merit_status merit_plan_scan(merit_dtype type, int64_t B, int64_t L, int64_t D, int64_t N, int64_t groups, int softplus,
                             merit_token_plan **out)
{
    if (!out) return MERIT_ERR_NULL;
    *out = nullptr;
    if (!type_ok(type) || B < 0 || L < 0 || D < 1 || N < 1 || groups < 1) return MERIT_ERR_INVALID_ARG;
    if (D % groups != 0) return MERIT_ERR_SHAPE;
    if (N > MERIT_SCAN_MAX_STATES || D > MAX_CHANNELS || B > MAX_ROWS || L > MAX_ROWS || too_large(B, L, D))
        return MERIT_ERR_UNSUPPORTED;
    merit_token_plan *pl = new_plan(SCAN, type);
    if (!pl) return MERIT_ERR_INVALID_ARG;
    ScanParams &p = pl->scan;
    p.B = B; p.L = L; p.D = (int)D; p.N = (int)N; p.G = (int)groups; p.Dg = (int)(D / groups);
    p.softplus = softplus != 0;
    p.type = type;
    pl->scan_back = p;
    scan_layout(p, false);
    scan_layout(pl->scan_back, true);
    const int64_t per = (int64_t)p.chunks * p.G * p.ctiles, lanes = (int64_t)D * scan_lpc(p.N), bc = groups * 2 * N;
    // (the last: launch_reduce_rows over A's gradient, 1024 threads for 64 sums)
    if (B > MAX_BLOCKS || D * (N + 2) > MAX_BLOCKS * 8 || B * per >= MAX_BLOCKS || cdiv(B * lanes, 256) >= MAX_BLOCKS ||
        (L > 0 && B > (MAX_BLOCKS * 256 - 256) / bc / L)) {
        delete pl;
        return MERIT_ERR_UNSUPPORTED;
    }
    *out = pl;
    return MERIT_OK;
}

merit_status merit_token_plan_destroy(merit_token_plan *plan)
{
    if (!plan) return MERIT_ERR_NULL;
    delete plan;
    return MERIT_OK;
}

merit_status merit_token_plan_workspace(const merit_token_plan *plan, merit_pass pass, int64_t *bytes)
{
    if (!plan || !bytes) return MERIT_ERR_NULL;
    *bytes = 0;
    if (plan->kind == DELTA || plan->kind == BLOCK) return mixer_workspace(plan, pass, bytes);
    if ((int)pass < 0 || (int)pass > 2 || (plan->kind == NORM && pass == MERIT_PASS_STEP)) return MERIT_ERR_INVALID_ARG;
    if (pass == MERIT_PASS_STEP) return MERIT_OK;
    const bool backward = pass == MERIT_PASS_BACKWARD;
    if (plan->kind == NORM) *bytes = norm_bytes(plan->norm, plan->type, backward);
    else if (plan->kind == CONV) *bytes = conv_bytes(plan->conv, plan->type, backward);
    else {
        const ScanParams &q = backward ? plan->scan_back : plan->scan;
        *bytes = 4 * (scan_chunk_floats(q) + (backward ? scan_part_bc(q) + scan_part_a(q) : 0));
    }
    return MERIT_OK;
}

merit_status merit_token_plan_kernel(const merit_token_plan *plan, merit_pass pass, const char **name)
{
    if (!plan || !name) return MERIT_ERR_NULL;
    *name = nullptr;
    if (plan->kind == DELTA || plan->kind == BLOCK) return mixer_kernel(plan, pass, name);
    if ((int)pass < 0 || (int)pass > 2 || (plan->kind == NORM && pass == MERIT_PASS_STEP)) return MERIT_ERR_INVALID_ARG;
    const bool backward = pass == MERIT_PASS_BACKWARD;
    if (plan->kind == NORM) {
        NormParams q = plan->norm;
        norm_layout(q, norm_vec(q, plan->type, [](int) { return true; }), backward);
        *name = q.rows_form ? (backward ? "merit_norm_rows_backward+merit_reduce_rows" : "merit_norm_rows")
                : q.slab    ? (backward ? "merit_norm_slab_backward+merit_reduce_rows" : "merit_norm_slab")
                            : (backward ? "merit_norm_sums+merit_norm_apply_backward+merit_reduce_rows"
                                        : "merit_norm_stats+merit_norm_apply");
    } else if (plan->kind == CONV) {
        *name = pass == MERIT_PASS_STEP ? "merit_cconv_step" : backward ? "merit_cconv_backward+merit_reduce_rows" : "merit_cconv";
    } else {
        const ScanParams &q = backward ? plan->scan_back : plan->scan;
        const bool split = q.chunks > 1;        // (then the workgroups are few: SCAN_FORWARD_BLOCKS is for unsplit sequences)
        const int64_t launches = split ? 2 : cdiv(q.B * q.G * q.ctiles, SCAN_FORWARD_BLOCKS);
        *name = pass == MERIT_PASS_STEP ? "merit_scan_token"
                : backward              ? (split ? "merit_scan_back_chunks+merit_scan_back+merit_scan_sum_bc+merit_reduce_rows"
                                                 : "merit_scan_back+merit_scan_sum_bc+merit_reduce_rows")
                : launches > 2          ? "merit_scan_tiles+merit_scan_tiles+merit_scan_tiles"
                : launches == 2         ? "merit_scan_tiles+merit_scan_tiles"
                                        : "merit_scan_tiles";
    }
    return MERIT_OK;
}

// ---- group norm ---------------------------------------------------------------------------------
merit_status merit_group_norm(const merit_token_plan *plan, const merit_group_norm_args *a, void *workspace,
                              int64_t workspace_bytes, void *stream)
{
    if (!plan || !a) return MERIT_ERR_NULL;
    if (plan->kind != NORM) return MERIT_ERR_INVALID_ARG;
    NormParams p = plan->norm;
    if (p.N == 0) return MERIT_OK;
    const bool some = p.S > 0;
    Views v{plan->type};
    p.x = v.rows(a->x, some);
    p.w = v.param(a->weight);
    p.b = v.param(a->bias);
    p.y = v.rows(a->y, some);
    p.mean = v.f32(a->mean);
    p.rstd = v.f32(a->rstd);
    if (v.st != MERIT_OK) return v.st;
    const int vec = norm_vec(p, plan->type, [&](int n) { return wide(p.x, p.N, p.S, n, plan->type) && wide(p.y, p.N, p.S, n, plan->type); });
    const int64_t need = 4 * norm_layout(p, vec, false);
    const merit_status st = scratch(need, workspace, workspace_bytes);
    if (st != MERIT_OK) return st;
    p.part = static_cast<float *>(workspace);
    return done(launch_norm(p, plan->type, static_cast<hipStream_t>(stream)));
}

merit_status merit_group_norm_backward(const merit_token_plan *plan, const merit_group_norm_backward_args *a, void *workspace,
                                       int64_t workspace_bytes, void *stream)
{
    if (!plan || !a) return MERIT_ERR_NULL;
    if (plan->kind != NORM) return MERIT_ERR_INVALID_ARG;
    NormParams p = plan->norm;
    const bool some = p.N > 0 && p.S > 0;
    Views v{plan->type};
    p.dy = v.rows(a->dy, some);
    p.x = v.rows(a->x, some);
    p.mean = v.f32(a->mean, some);
    p.rstd = v.f32(a->rstd, some);
    p.w = v.param(a->weight);
    p.b = v.param(a->bias);
    p.dx = v.rows(a->dx, some);
    p.dw = v.f32(a->dweight);
    p.db = v.f32(a->dbias);
    if (v.st != MERIT_OK) return v.st;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (!some) {                                        // no gradient from nothing: zeros
        if (!p.dw && !p.db) return MERIT_OK;
        ReduceParams r = {};
        r.nseg = 2;
        r.seg[0] = {p.db, 0, p.C};
        r.seg[1] = {p.dw, 0, p.C};
        return done(launch_reduce_rows(r, s));
    }
    const int vec = norm_vec(p, plan->type, [&](int n) {
        return wide(p.x, p.N, p.S, n, plan->type) && wide(p.dy, p.N, p.S, n, plan->type) && wide(p.dx, p.N, p.S, n, plan->type);
    });
    const int64_t need = 4 * norm_layout(p, vec, true);
    const merit_status st = scratch(need, workspace, workspace_bytes);
    if (st != MERIT_OK) return st;
    p.part = static_cast<float *>(workspace);
    return done(launch_norm_backward(p, plan->type, s));
}

// ---- causal convolution ------------------------------------------------------------------------------
merit_status merit_causal_conv(const merit_token_plan *plan, const merit_causal_conv_args *a, void *, int64_t, void *stream)
{
    if (!plan || !a) return MERIT_ERR_NULL;
    if (plan->kind != CONV) return MERIT_ERR_INVALID_ARG;
    CconvParams p = plan->conv;
    if (p.B == 0) return MERIT_OK;
    Views v{plan->type};
    p.x = v.rows(a->x, p.L > 0);
    p.w = v.param(a->weight, true);
    p.b = v.param(a->bias);
    p.init = v.rows(a->init, false);
    p.lens = v.lens(a->lens);
    p.y = v.rows(a->y, p.L > 0);
    p.fin = v.rows(a->final, false);
    if (v.st != MERIT_OK) return v.st;
    const int vec = CONV_VEC;
    const bool fits = p.D % vec == 0 && wide(p.x, p.B, p.L, vec, plan->type) && wide(p.y, p.B, p.L, vec, plan->type) &&
                      wide(p.init, p.B, p.K - 1, vec, plan->type) && wide(p.fin, p.B, p.K - 1, vec, plan->type);
    conv_layout(p, fits ? vec : 1, false);
    return done(launch_cconv(p, plan->type, static_cast<hipStream_t>(stream)));
}

merit_status merit_causal_conv_backward(const merit_token_plan *plan, const merit_causal_conv_backward_args *a, void *workspace,
                                        int64_t workspace_bytes, void *stream)
{
    if (!plan || !a) return MERIT_ERR_NULL;
    if (plan->kind != CONV) return MERIT_ERR_INVALID_ARG;
    CconvParams p = plan->conv;
    const bool some = p.B > 0 && p.L > 0;
    Views v{plan->type};
    p.dy = v.rows(a->dy, some);
    p.x = v.rows(a->x, some);
    p.w = v.param(a->weight, true);
    p.b = v.param(a->bias);
    p.init = v.rows(a->init, false);
    p.lens = v.lens(a->lens);
    p.dfin = v.rows(a->dfinal, false);
    p.dx = v.rows(a->dx, some);
    p.dw = v.f32(a->dweight);
    p.db = v.f32(a->dbias);
    p.dinit = v.rows(a->dinit, false);
    if (v.st != MERIT_OK) return v.st;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (p.B == 0) {
        if (!p.dw && !p.db) return MERIT_OK;
        ReduceParams r = {};
        r.nseg = 2;
        r.seg[0] = {p.dw, 0, (int64_t)p.K * p.D};
        r.seg[1] = {p.db, 0, p.D};
        return done(launch_reduce_rows(r, s));
    }
    const int vec = CONV_VEC;
    const bool fits = p.D % vec == 0 && wide(p.x, p.B, p.L, vec, plan->type) && wide(p.dy, p.B, p.L, vec, plan->type) && wide(p.dx, p.B, p.L, vec, plan->type) &&
                      wide(p.init, p.B, p.K - 1, vec, plan->type);
    const int64_t need = 4 * conv_layout(p, fits ? vec : 1, true);
    const merit_status st = scratch(need, workspace, workspace_bytes);
    if (st != MERIT_OK) return st;
    p.part = static_cast<float *>(workspace);
    return done(launch_cconv_backward(p, plan->type, s));
}

merit_status merit_causal_conv_step(const merit_token_plan *plan, const merit_causal_conv_step_args *a, void *, int64_t,
                                    void *stream)
{
    if (!plan || !a) return MERIT_ERR_NULL;
    if (plan->kind != CONV) return MERIT_ERR_INVALID_ARG;
    CconvParams p = plan->conv;
    if (p.B == 0) return MERIT_OK;
    Views v{plan->type};
    p.init = v.rows(a->kept, p.K > 1);
    p.x = v.rows(a->x);
    p.w = v.param(a->weight, true);
    p.b = v.param(a->bias);
    p.y = v.rows(a->y);
    p.fin = v.rows(a->kept_out, p.K > 1);
    if (v.st != MERIT_OK) return v.st;
    const int vec = CONV_VEC;
    const bool fits = p.D % vec == 0 && wide(p.x, p.B, 1, vec, plan->type) && wide(p.y, p.B, 1, vec, plan->type) && wide(p.init, p.B, p.K - 1, vec, plan->type) &&
                      wide(p.fin, p.B, p.K - 1, vec, plan->type);
    p.vec = fits ? vec : 1;
    return done(launch_cconv_step(p, plan->type, static_cast<hipStream_t>(stream)));
}

// ---- scan -----------------------------------------------------------------------------------------------
merit_status merit_scan(const merit_token_plan *plan, const merit_scan_args *a, void *workspace, int64_t workspace_bytes, void *stream)
{
    if (!plan || !a) return MERIT_ERR_NULL;
    if (plan->kind != SCAN) return MERIT_ERR_INVALID_ARG;
    ScanParams p = plan->scan;
    if (p.B == 0) return MERIT_OK;
    const bool some = p.L > 0;
    Views v{plan->type};
    p.x = v.rows(a->x, some);
    p.dt = v.rows(a->dt, some);
    p.A = v.f32(a->A, true);
    p.Bm = v.rows(a->B, some);
    p.Cm = v.rows(a->C, some);
    p.skip = v.f32(a->skip);
    p.z = v.rows(a->z, false);
    p.dt_bias = v.f32(a->dt_bias);
    p.h0 = v.f32(a->h0);
    p.lens = v.lens(a->lens);
    p.y = v.rows(a->y, some);
    p.h_last = v.f32(a->h_last);
    p.states = v.f32(a->states);
    if (v.st != MERIT_OK) return v.st;
    const merit_status st = scratch(4 * scan_chunk_floats(p), workspace, workspace_bytes);
    if (st != MERIT_OK) return st;
    p.chunk_dt = static_cast<float *>(workspace);
    p.chunk_h = p.chunk_dt + (p.chunks > 1 ? p.B * p.chunks * p.D : 0);
    return done(launch_scan(p, static_cast<hipStream_t>(stream)));
}

merit_status merit_scan_backward(const merit_token_plan *plan, const merit_scan_backward_args *a, void *workspace,
                                 int64_t workspace_bytes, void *stream)
{
    if (!plan || !a) return MERIT_ERR_NULL;
    if (plan->kind != SCAN) return MERIT_ERR_INVALID_ARG;
    ScanParams p = plan->scan_back;
    const bool some = p.B > 0 && p.L > 0;
    Views v{plan->type};
    p.dy = v.rows(a->dy, some);
    p.x = v.rows(a->x, some);
    p.dt = v.rows(a->dt, some);
    p.A = v.f32(a->A, true);
    p.Bm = v.rows(a->B, some);
    p.Cm = v.rows(a->C, some);
    p.states = v.f32(a->states, some);
    p.skip = v.f32(a->skip);
    p.z = v.rows(a->z, false);
    p.dt_bias = v.f32(a->dt_bias);
    p.lens = v.lens(a->lens);
    p.dh_last = v.f32(a->dh_last);
    p.dx = v.rows(a->dx, some);
    p.ddt = v.rows(a->ddt, some);
    p.dB = v.rows(a->dB, some);
    p.dC = v.rows(a->dC, some);
    p.dz = v.rows(a->dz, some && p.z.data);
    p.dA = v.f32(a->dA, true);
    p.dskip = v.f32(a->dskip);
    p.ddt_bias = v.f32(a->ddt_bias);
    p.dh0 = v.f32(a->dh0);
    if (v.st != MERIT_OK) return v.st;
    const int64_t need = 4 * (scan_part_bc(p) + scan_part_a(p) + scan_chunk_floats(p));
    const merit_status st = scratch(need, workspace, workspace_bytes);
    if (st != MERIT_OK) return st;
    p.part_a = static_cast<float *>(workspace);
    p.part_bc = p.part_a + scan_part_a(p);
    p.chunk_dt = p.part_bc + scan_part_bc(p);
    p.chunk_h = p.chunk_dt + (p.chunks > 1 ? p.B * p.chunks * p.D : 0);
    return done(launch_scan_backward(p, static_cast<hipStream_t>(stream)));
}

merit_status merit_scan_step(const merit_token_plan *plan, const merit_scan_step_args *a, void *, int64_t, void *stream)
{
    if (!plan || !a) return MERIT_ERR_NULL;
    if (plan->kind != SCAN) return MERIT_ERR_INVALID_ARG;
    ScanParams p = plan->scan;
    if (p.B == 0) return MERIT_OK;
    Views v{plan->type};
    p.h0 = v.f32(a->h, true);
    p.x = v.rows(a->x);
    p.dt = v.rows(a->dt);
    p.A = v.f32(a->A, true);
    p.Bm = v.rows(a->B);
    p.Cm = v.rows(a->C);
    p.skip = v.f32(a->skip);
    p.z = v.rows(a->z, false);
    p.dt_bias = v.f32(a->dt_bias);
    p.y = v.rows(a->y);
    p.h_last = v.f32(a->h_out, true);
    if (v.st != MERIT_OK) return v.st;
    return done(launch_scan_step(p, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
