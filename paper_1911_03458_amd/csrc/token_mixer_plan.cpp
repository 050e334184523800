// Plans and entry points of the gated delta rule and of the norms before and after a block (include/merit_tokens.h): what is
// accepted, how a pass is split into workgroups, how much scratch memory it takes.  Host code only.
#include "token_plan.h"

#include <algorithm>

using namespace merit;

namespace {

Rows rows_of(Views &v, const merit_view &view, int type, bool required)
{
    const int own = v.type;
    v.type = type;
    const Rows r = v.rows(view, required);
    v.type = own;
    return r;
}

// ---- gated delta rule ------------------------------------------------------------------------
// Segments of a sequence's chunks side by side, where heads and sequences leave compute units idle: what a segment does to a state is
// found first (a launch for all but the last, and a product a segment), then each goes from its own first state.  An estimate, in us:
// a chunk takes a workgroup of 16, 32 or 64 columns 4.2, 4.9 or 5.9, and without results 3.0, 3.6 or 3.7; launches 10, products 3.
// Those are times of states of 128 x 128, bfloat16, up to 256 workgroups, and stand for the others too: it is their ratios that
// decide.  16 heads of 8191 tokens in 1, 2, 3, 4, 5, 6, 8 and 12 segments take 551, 460, 331, 273, 228, 268, 222 and 261 us
// (merit_delta_prepare, 41, not included).  Whole calls in one piece against what this chooses: 16 heads of 8191, 128 x 128, fp32 1043 against
// 434, binary16 826 against 338; 8 heads of 8192, 64 x 64, fp32 632 against 144; 16 heads of 1024, 32 x 32, 73 against 51; 64
// heads of 16384, 64 x 64, 1607 against 1113.  Not for less than a fifth, which leaves more than about 300 workgroups of 64 columns
// in one piece: the launch that joins segments, 512 threads for 16 columns of a head, is a small one.
void delta_segments(DeltaParams &p)
{
    const int64_t heads = p.B * p.H;
    auto turn = [](int64_t groups, int Dv, int more) {
        const int w = delta_width(groups, Dv, more);
        const double us = more ? w == 16 ? 3.0 : w == 32 ? 3.6 : 3.7 : w == 16 ? 4.2 : w == 32 ? 4.9 : 5.9;
        return us * (double)cdiv(groups * delta_slices(w, Dv, more), 256);
    };
    p.segments = 1;
    p.seg_chunks = p.n > 0 ? p.n : 1;
    if (heads < 1 || heads > 256) return;
    double least = 0.8 * p.n * turn(heads, p.Dv, 0);
    for (int s = 2; s <= 16; ++s) {
        const int chunks = (int)cdiv(p.n, s);
        if (chunks < 1 || cdiv(p.n, chunks) != s) continue;
        const double us = chunks * (turn(heads * s, p.Dv, 0) + turn(heads * (s - 1), p.Dv, p.Dk)) + 10.0 + 3.0 * (s - 2);
        if (us < least) {
            least = us;
            p.segments = s;
            p.seg_chunks = chunks;
        }
    }
}
// Floats that the forward pass keeps of a chunk of a head
int64_t delta_kept(const DeltaParams &p) { return cdiv(DELTA_PREPARED_FLOATS + (int64_t)(p.Dk + MERIT_DELTA_CHUNK) * p.Dv, 4) * 4; }
// Scratch memory.  Forward: what the chunks' tokens do to each other (a call that keeps states has it there instead), segments' states.  Backward: x, the
// gradients of the states, and the value heads' parts of dq and dk; each a multiple of 16 bytes but the last.
struct DeltaScratch {
    int64_t seg, dx, ds, part, bytes;
};
DeltaScratch delta_scratch(const DeltaParams &p, bool backward)
{
    const int64_t chunks = p.B * p.n * p.H;
    DeltaScratch s = {};
    if (!backward) {
        s.seg = chunks * DELTA_PREPARED_FLOATS * 4;
        s.bytes = s.seg + (p.segments > 1 ? delta_segment_floats(p, p.segments, p.segments - 2) * 4 : 0);
        return s;
    }
    s.ds = s.dx + chunks * MERIT_DELTA_CHUNK * p.Dv * 4;
    s.part = s.ds + (chunks * p.Dk * p.Dv * 4 + 15) / 16 * 16;
    s.bytes = s.part + (p.each > 1 ? 2 * p.B * p.L * p.H * p.Dk * 4 : 0);
    return s;
}
void delta_gates(Views &v, DeltaParams &p, const merit_view &g, const merit_view &beta)
{
    p.g = rows_of(v, g, MERIT_F32, false);
    p.beta_f32 = beta.dtype == MERIT_F32;
    p.beta = rows_of(v, beta, p.beta_f32 ? MERIT_F32 : v.type, true);
}
bool in_16_bytes(const Rows &r, int64_t n0, int64_t n1, int type) { return wide(r, n0, n1, 16 / elem_bytes(type), type); }
bool address_16(const void *a) { return reinterpret_cast<uintptr_t>(a) % 16 == 0; }

// ---- the norms before and after a block -----------------------------------------------------
// The threads of a row for `vec` channels each: a run of lanes up to 64 vectors, else a workgroup.
void block_layout(BlockNormParams &p, int vec, bool backward)
{
    p.vec = vec;
    const int cu = p.C / vec;
    p.lanes = 0;
    p.units = 1;
    p.threads = cu <= 256 ? 256 : 512;
    if (cu <= 64) {
        p.lanes = 1;
        while (p.lanes < cu) p.lanes *= 2;
    }
    while (p.threads * p.units < cu) p.units *= 2;
    const int64_t at_once = p.lanes ? 256 / p.lanes : 1;
    // No more workgroups than run at once, by the registers that each takes: forward 1024 wavefronts of 4 against twice as many,
    // 8 x 2048 rows of 2048, both norms, 49 against 51 us; backward 512 against 768, the same rows, 85 against 99 us, and 1024
    // against 512 where there is an after-norm only, 262144 rows of 128, 73 against 81 us.
    const int64_t fours = backward && p.before ? 512 : 1024;
    const int64_t most = fours * 256 / p.threads;
    p.blocks = cdiv(p.rows, at_once);
    if (p.blocks > most) p.blocks = most;
}
template <typename F> int block_vec(const BlockNormParams &p, F &&fits)
{
    const int most = 16 / elem_bytes(p.type);
    for (int vec : {most, 2})
        if (p.C % vec == 0 && fits(vec)) return vec;
    return 1;
}
bool block_rows(const BlockNormParams &p, const Rows &r, int vec, int type)
{
    return wide(r, p.B, p.L, type == MERIT_F32 && vec > 4 ? 4 : vec, type);
}
int64_t block_bytes(const BlockNormParams &p)
{
    int64_t most = 0;
    for (int vec : {16 / elem_bytes(p.type), 2, 1}) {
        if (p.C % vec) continue;
        BlockNormParams q = p;
        block_layout(q, vec, true);
        const int64_t n = q.blocks * 5 * p.C * 4;
        if (n > most) most = n;
    }
    return most;
}

}  // namespace

namespace merit {

merit_status mixer_workspace(const merit_token_plan *plan, merit_pass pass, int64_t *bytes)
{
    if ((int)pass < 0 || (int)pass > 2 || (plan->kind == BLOCK && pass == MERIT_PASS_STEP)) return MERIT_ERR_INVALID_ARG;
    if (pass == MERIT_PASS_STEP) return MERIT_OK;
    const bool backward = pass == MERIT_PASS_BACKWARD;
    if (plan->kind == DELTA) *bytes = delta_scratch(plan->delta, backward).bytes;
    else *bytes = backward ? block_bytes(plan->block) : 0;
    return MERIT_OK;
}

merit_status mixer_kernel(const merit_token_plan *plan, merit_pass pass, const char **name)
{
    if ((int)pass < 0 || (int)pass > 2 || (plan->kind == BLOCK && pass == MERIT_PASS_STEP)) return MERIT_ERR_INVALID_ARG;
    const bool backward = pass == MERIT_PASS_BACKWARD;
    if (plan->kind == BLOCK)
        *name = backward ? "merit_block_norm_rows_backward+merit_reduce_rows" : "merit_block_norm_rows";
    else
        *name = pass == MERIT_PASS_STEP   ? "merit_delta_token"
                : !backward               ? plan->delta.segments < 2   ? "merit_delta_prepare+merit_delta_chunks"
                                            : plan->delta.segments > 2 ? "merit_delta_prepare+merit_delta_chunks+merit_delta_join+merit_delta_chunks"
                                                                       : "merit_delta_prepare+merit_delta_chunks+merit_delta_chunks"
                : plan->delta.each > 1    ? "merit_delta_back_chunks+merit_delta_grads+merit_delta_sum_heads"
                                          : "merit_delta_back_chunks+merit_delta_grads";
    return MERIT_OK;
}

}  // namespace merit

extern "C" {

merit_status merit_plan_delta_rule(merit_dtype type, int64_t B, int64_t L, int64_t heads, int64_t key_heads, int64_t Dk, int64_t Dv,
                                   double scale, int normalize, merit_token_plan **out)
{
    if (!out) return MERIT_ERR_NULL;
    *out = nullptr;
    if (!type_ok(type) || B < 0 || L < 0 || heads < 1 || key_heads < 1 || Dk < 1 || Dv < 1 || !std::isfinite((float)scale))
        return MERIT_ERR_INVALID_ARG;
    if (heads % key_heads != 0) return MERIT_ERR_SHAPE;
    if (Dk > MERIT_DELTA_MAX_KEYS || Dv > MAX_CHANNELS || heads > MAX_CHANNELS / Dv || heads > MAX_CHANNELS / Dk || B > MAX_ROWS ||
        L > MAX_ROWS || too_large(B, L, heads * (Dk + Dv)))
        return MERIT_ERR_UNSUPPORTED;
    const int64_t n = cdiv(L, MERIT_DELTA_CHUNK);
    // workgroups of every pass, in units of 256 threads: of 512 a chunk, of 512 for at most 64 columns (fewer columns only in launches of up
    // to 256 workgroups), of 256 for 16 columns of a token; the sum over heads, a thread a value; states of all chunks
    const int64_t most = std::max(2 * std::max(n, cdiv(Dv, 64)), cdiv(Dv, 16));
    if (B > MAX_BLOCKS / heads || B * heads * most >= MAX_BLOCKS || too_large(B * heads, n + 1, (Dk + MERIT_DELTA_CHUNK) * Dv + MERIT_DELTA_KEPT) ||
        (L > 0 && B > MAX_BLOCKS / L * 256 / (key_heads * Dk)))
        return MERIT_ERR_UNSUPPORTED;
    merit_token_plan *pl = new_plan(DELTA, type);
    if (!pl) return MERIT_ERR_INVALID_ARG;
    DeltaParams &p = pl->delta;
    p.B = B; p.L = L;
    p.H = (int)heads; p.K = (int)key_heads; p.each = (int)(heads / key_heads);
    p.Dk = (int)Dk; p.Dv = (int)Dv;
    p.scale = (float)scale;
    p.unit = normalize != 0;
    p.type = type;
    p.n = (int)n;
    delta_segments(p);
    *out = pl;
    return MERIT_OK;
}

merit_status merit_plan_block_norm(merit_dtype type, merit_dtype stream, int64_t B, int64_t L, int64_t C, double eps, int layer,
                                   merit_act act, int after, int before, merit_token_plan **out)
{
    if (!out) return MERIT_ERR_NULL;
    *out = nullptr;
    if (!type_ok(type) || (stream != type && stream != MERIT_F32) || (int)act < 0 || (int)act > 3 || B < 0 || L < 0 || C < 1 ||
        !(eps >= 0.0) || !std::isfinite((float)eps) || !(after || before))
        return MERIT_ERR_INVALID_ARG;
    if (C > MERIT_BLOCK_NORM_MAX_CHANNELS || B > MAX_ROWS || L > MAX_ROWS || (L > 0 && B > MAX_ROWS / L)) return MERIT_ERR_UNSUPPORTED;
    merit_token_plan *pl = new_plan(BLOCK, type);
    if (!pl) return MERIT_ERR_INVALID_ARG;
    BlockNormParams &p = pl->block;
    p.B = B; p.L = L; p.rows = B * L;
    p.C = (int)C;
    p.eps = (float)eps;
    p.layer = layer != 0;
    p.act = act;
    p.after = after != 0;
    p.before = before != 0;
    p.type = type;
    p.stream = stream;
    *out = pl;
    return MERIT_OK;
}

// ---- gated delta rule ---------------------------------------------------------------------------
merit_status merit_delta_rule(const merit_token_plan *plan, const merit_delta_rule_args *a, void *workspace, int64_t workspace_bytes,
                              void *stream)
{
    if (!plan || !a) return MERIT_ERR_NULL;
    if (plan->kind != DELTA) return MERIT_ERR_INVALID_ARG;
    DeltaParams p = plan->delta;
    if (p.B == 0) return MERIT_OK;
    const bool some = p.L > 0;
    Views v{plan->type};
    p.q = v.rows(a->q, some);
    p.k = v.rows(a->k, some);
    p.v = v.rows(a->v, some);
    if (some) delta_gates(v, p, a->g, a->beta);
    p.h0 = v.f32(a->h0);
    p.lens = v.lens(a->lens);
    p.y = v.rows(a->y, some);
    p.h_last = v.f32(a->h_last);
    p.states = v.f32(a->states);
    if (v.st != MERIT_OK) return v.st;
    if (p.states && reinterpret_cast<uintptr_t>(p.states) % 16 != 0) return MERIT_ERR_ALIGNMENT;
    const merit_status st = scratch(delta_scratch(p, false).bytes, workspace, workspace_bytes);
    if (st != MERIT_OK) return st;
    p.prep = p.states ? p.states : static_cast<float *>(workspace);
    p.seg_state = static_cast<float *>(workspace) + delta_scratch(p, false).seg / 4;
    p.prep_stride = p.states ? delta_kept(p) : DELTA_PREPARED_FLOATS;
    p.wide_qk = p.Dk % 8 == 0 && in_16_bytes(p.q, p.B, p.L, p.type) && in_16_bytes(p.k, p.B, p.L, p.type);
    return done(launch_delta(p, static_cast<hipStream_t>(stream)));
}

merit_status merit_delta_rule_backward(const merit_token_plan *plan, const merit_delta_rule_backward_args *a, void *workspace,
                                       int64_t workspace_bytes, void *stream)
{
    if (!plan || !a) return MERIT_ERR_NULL;
    if (plan->kind != DELTA) return MERIT_ERR_INVALID_ARG;
    DeltaParams p = plan->delta;
    if (p.B == 0) return MERIT_OK;
    const bool some = p.L > 0;
    Views v{plan->type};
    p.dy = v.rows(a->dy, some);
    p.q = v.rows(a->q, some);
    p.k = v.rows(a->k, some);
    if (some) delta_gates(v, p, a->g, a->beta);
    p.states = v.f32(a->states, some);
    p.lens = v.lens(a->lens);
    p.dh_last = v.f32(a->dh_last);
    p.dq = v.rows(a->dq, some);
    p.dk = v.rows(a->dk, some);
    p.dv = v.rows(a->dv, some);
    p.dg = rows_of(v, a->dg, MERIT_F32, false);
    p.dbeta = rows_of(v, a->dbeta, MERIT_F32, some);
    p.dh0 = v.f32(a->dh0);
    if (v.st != MERIT_OK) return v.st;
    if (some && reinterpret_cast<uintptr_t>(p.states) % 16 != 0) return MERIT_ERR_ALIGNMENT;
    const DeltaScratch at = delta_scratch(p, true);
    const merit_status st = scratch(at.bytes, workspace, workspace_bytes);
    if (st != MERIT_OK) return st;
    char *const base = static_cast<char *>(workspace);
    p.dx = reinterpret_cast<float *>(base + at.dx);
    p.ds = reinterpret_cast<float *>(base + at.ds);
    p.part = p.each > 1 ? reinterpret_cast<float *>(base + at.part) : nullptr;
    p.prep = p.states;
    p.prep_stride = delta_kept(p);
    p.wide_qk = p.Dk % 8 == 0 && in_16_bytes(p.q, p.B, p.L, p.type) && in_16_bytes(p.k, p.B, p.L, p.type);
    p.wide_out = p.Dk % 8 == 0 && in_16_bytes(p.dq, p.B, p.L, p.type) && in_16_bytes(p.dk, p.B, p.L, p.type);
    p.wide_v = p.Dv % 8 == 0 && in_16_bytes(p.dy, p.B, p.L, p.type);
    return done(launch_delta_backward(p, static_cast<hipStream_t>(stream)));
}

merit_status merit_delta_rule_step(const merit_token_plan *plan, const merit_delta_rule_step_args *a, void *, int64_t, void *stream)
{
    if (!plan || !a) return MERIT_ERR_NULL;
    if (plan->kind != DELTA) return MERIT_ERR_INVALID_ARG;
    DeltaParams p = plan->delta;
    if (p.B == 0) return MERIT_OK;
    Views v{plan->type};
    p.h0 = v.f32(a->h, true);
    p.q = v.rows(a->q);
    p.k = v.rows(a->k);
    p.v = v.rows(a->v);
    delta_gates(v, p, a->g, a->beta);
    p.y = v.rows(a->y);
    p.h_last = v.f32(a->h_out, true);
    if (v.st != MERIT_OK) return v.st;
    p.wide_state = p.Dv % 4 == 0 && address_16(p.h0) && address_16(p.h_last);
    return done(launch_delta_step(p, static_cast<hipStream_t>(stream)));
}

// ---- the norms before and after a block -----------------------------------------------------------
merit_status merit_block_norm(const merit_token_plan *plan, const merit_block_norm_args *a, void *, int64_t, void *stream)
{
    if (!plan || !a) return MERIT_ERR_NULL;
    if (plan->kind != BLOCK) return MERIT_ERR_INVALID_ARG;
    BlockNormParams p = plan->block;
    if (p.rows == 0) return MERIT_OK;
    Views v{plan->type};
    p.x = v.rows(a->x);
    p.z = v.rows(a->z, false);
    p.r = rows_of(v, a->r, p.stream, false);
    p.aw = v.param(a->after_weight);
    p.ab = v.param(a->after_bias);
    p.scale = v.param(a->scale);
    p.bw = v.param(a->before_weight);
    p.bb = v.param(a->before_bias);
    p.out = rows_of(v, a->out, p.stream, true);
    p.n = v.rows(a->n, p.before);
    p.am = v.f32(a->after_mean);
    p.ar = v.f32(a->after_rstd);
    p.bm = v.f32(a->before_mean);
    p.br = v.f32(a->before_rstd);
    if (v.st != MERIT_OK) return v.st;
    if ((!p.after && (p.aw.data || p.ab.data)) || (!p.before && (p.bw.data || p.bb.data || p.n.data))) return MERIT_ERR_INVALID_ARG;
    const int vec = block_vec(p, [&](int n) {
        return block_rows(p, p.x, n, p.type) && block_rows(p, p.z, n, p.type) && block_rows(p, p.n, n, p.type) &&
               block_rows(p, p.r, n, p.stream) && block_rows(p, p.out, n, p.stream);
    });
    block_layout(p, vec, false);
    return done(launch_block_norm(p, static_cast<hipStream_t>(stream)));
}

merit_status merit_block_norm_backward(const merit_token_plan *plan, const merit_block_norm_backward_args *a, void *workspace,
                                       int64_t workspace_bytes, void *stream)
{
    if (!plan || !a) return MERIT_ERR_NULL;
    if (plan->kind != BLOCK) return MERIT_ERR_INVALID_ARG;
    BlockNormParams p = plan->block;
    const bool some = p.rows > 0;
    Views v{plan->type};
    p.dout = rows_of(v, a->dout, p.stream, false);
    p.dn = v.rows(a->dn, some && p.before);
    p.x = v.rows(a->x, some);
    p.z = v.rows(a->z, false);
    p.r = rows_of(v, a->r, p.stream, false);
    p.aw = v.param(a->after_weight);
    p.ab = v.param(a->after_bias);
    p.scale = v.param(a->scale);
    p.bw = v.param(a->before_weight);
    p.am = v.f32(a->after_mean, some && p.after && p.layer);
    p.ar = v.f32(a->after_rstd, some && p.after);
    p.bm = v.f32(a->before_mean, some && p.before && p.layer);
    p.br = v.f32(a->before_rstd, some && p.before);
    p.dx = v.rows(a->dx, some);
    p.dz = v.rows(a->dz, some && p.z.data);
    p.dr = rows_of(v, a->dr, p.stream, false);
    p.daw = v.f32(a->dafter_weight);
    p.dab = v.f32(a->dafter_bias);
    p.dscale = v.f32(a->dscale);
    p.dbw = v.f32(a->dbefore_weight);
    p.dbb = v.f32(a->dbefore_bias);
    if (v.st != MERIT_OK) return v.st;
    if ((!p.after && (p.aw.data || p.ab.data || p.daw || p.dab)) || (!p.before && (p.bw.data || p.dbw || p.dbb || p.dn.data)) ||
        (!p.z.data && p.dz.data))
        return MERIT_ERR_INVALID_ARG;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if (!some) {                                        // no gradient from nothing: zeros
        ReduceParams r = {};
        for (float *o : {p.daw, p.dab, p.dscale, p.dbw, p.dbb})
            if (o) r.seg[r.nseg++] = {o, 0, p.C};
        return r.nseg ? done(launch_reduce_rows(r, s)) : MERIT_OK;
    }
    const int vec = block_vec(p, [&](int n) {
        for (const Rows *r : {&p.x, &p.z, &p.dn, &p.dx, &p.dz})
            if (!block_rows(p, *r, n, p.type)) return false;
        for (const Rows *r : {&p.dout, &p.r, &p.dr})
            if (!block_rows(p, *r, n, p.stream)) return false;
        return true;
    });
    block_layout(p, vec, true);
    const merit_status st = scratch(p.blocks * 5 * p.C * 4, workspace, workspace_bytes);
    if (st != MERIT_OK) return st;
    p.part = static_cast<float *>(workspace);
    return done(launch_block_norm_backward(p, s));
}

}  // extern "C"
