// C ABI of the layer of experts: host-side validation and launches (kernels in duo_moe.h).
#include "../../include/duo_verify.h"

#include "duo_internal.h"
#include "duo_moe.h"

namespace {

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool off4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }
size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }

int check_moe(const duo_moe_config* c) {
    if (!c) return DUO_ERR_NULL;
    static_assert(MOE_MAX_EXPERTS == DUO_MOE_MAX_EXPERTS && MOE_MAX_TOP == DUO_MOE_MAX_TOP && MOE_MAX_ROWS == DUO_MAX_ROWS, "what the kernels are laid out for");
    if (c->d_model < 64 || c->d_model % 64 || c->d_model > 8192 || c->d_ff < 32 || c->d_ff % 32 || c->d_ff > DUO_SCALED_MAX_K) return DUO_ERR_SHAPE;
    if (c->n_experts < 1 || c->n_experts > DUO_MOE_MAX_EXPERTS || c->top_k < 1 || c->top_k > DUO_MOE_MAX_TOP || c->top_k > c->n_experts) return DUO_ERR_SHAPE;
    if ((c->scaled != 0 && c->scaled != 1) || (c->renormalise != 0 && c->renormalise != 1)) return DUO_ERR_ARG;
    return DUO_OK;
}

size_t matrix_bytes(const duo_moe_config* c, int N, int K) { return c->scaled ? Narrow::bytes(N, K) : Wide::bytes(N, K); }
size_t expert_bytes(const duo_moe_config* c) { return 2 * matrix_bytes(c, c->d_ff, c->d_model) + matrix_bytes(c, c->d_model, c->d_ff); }

int up128(int n) { return (n + 127) / 128 * 128; }

struct MoeLayout {  // of the workspace
    size_t chosen, share, logits, hidden, partial, total;
};
MoeLayout layout_of(const duo_moe_config* c, int rows) {
    MoeLayout l{};
    size_t at = 0;
    const size_t entries = (size_t)rows * c->top_k;
    l.chosen = at, at += up16(4 * entries);
    l.share = at, at += up16(4 * entries);
    l.logits = at, at += up16(8 * (size_t)rows * c->n_experts * logit_parts(c->d_model));
    l.hidden = at, at += 4 * entries * up128(c->d_ff);
    l.partial = at, at += c->top_k > 1 ? 4 * entries * c->d_model : 0;
    l.total = at;
    return l;
}

int most_active(const MoeArgs& a) { return a.n_experts < a.rows * a.top ? a.n_experts : a.rows * a.top; }

template <class W, int MT, int NW, int PF>
void launch_gate_up(const MoeArgs& a, hipStream_t s) {
    duo_internal_prof(DUO_PROF_MOE_GATEUP);
    DUO_LAUNCH((moe_gate_up_kernel<W, MT, NW, PF>), dim3(a.ff / 16, most_active(a)), dim3(64 * NW), s, a);
}
template <class W, int MT, int NB, int NW, int PF>
void launch_down(const MoeArgs& a, hipStream_t s) {
    const dim3 grid(a.d / 16 / NB, most_active(a));
    duo_internal_prof(DUO_PROF_MOE_DOWN);
    if (a.top == 1) {
        DUO_LAUNCH((moe_down_kernel<W, MT, NB, NW, PF, true>), grid, dim3(64 * NW), s, a);
        return;
    }
    DUO_LAUNCH((moe_down_kernel<W, MT, NB, NW, PF, false>), grid, dim3(64 * NW), s, a);
    duo_internal_prof(DUO_PROF_MOE_DOWN);
    DUO_LAUNCH(moe_combine_kernel, dim3((a.d + 1023) / 1024, a.rows), dim3(256), s, a);
}
// Experts of two or three tiles of rows.  us with four bands for four waves, two for eight, one for eight: 60 rows, 4 of 8 experts, 4096 x 2048: 29, 48, 84;
// 64 rows, 2 of 4 experts, 2048 x 2816: 26, 19, 31; 32 rows, 2 experts of 896 x 6816 (two tiles): 35, 33, 29.
template <class W, int MT>
void launch_down_tiles(const MoeArgs& a, hipStream_t s) {
    if (most_active(a) * a.d > 12288) launch_down<W, MT, 4, 4, 1>(a, s);
    else if (most_active(a) * a.d > 4096) launch_down<W, MT, 2, 8, 1>(a, s);
    else launch_down<W, MT, 1, 8, 1>(a, s);
}
// By the rows an expert has where all have as many: the host does not know how many chose it.  Up to 12 hardly an expert has more than 16 where rows choose
// at random, and one tile of rows it is, over an expert's matrices once for every 16 rows where it has more (80 rows that all chose the same 4 of 128
// experts of 2048 x 1408 in 8 bits: 121 us for the products, and 172 where 115 experts are chosen).  80 rows, two choices of 8 experts (20 each) 102 us like this, 68 with two tiles; of 16 (10 each) 50, 52.  40 rows each: two tiles 29 us,
// three 21, five 22.
template <class W>
void launch_products(const MoeArgs& a, hipStream_t s) {
    const int each = a.rows * a.top / a.n_experts;
    if (each <= 12 || a.rows <= 16) {
        launch_gate_up<W, 1, 4, 2>(a, s);
        // four bands for two waves where that makes enough workgroups (128 experts of 4096 x 1536 in 8 bits: 145 us, two bands for four waves 171), two
        // for four where not (two experts of 4096 x 14336: 22, four bands 30), and one for eight where the outputs are few (two experts of 320 x 7680: 9.4, two bands 14.7)
        if (most_active(a) * a.d > 16384) launch_down<W, 1, 4, 2, 1>(a, s);
        else if (most_active(a) * a.d > 4096) launch_down<W, 1, 2, 4, 2>(a, s);
        else launch_down<W, 1, 1, 8, 1>(a, s);
    } else if (each <= 28) {
        launch_gate_up<W, 2, 4, 1>(a, s);
        launch_down_tiles<W, 2>(a, s);
    } else {
        launch_gate_up<W, 3, 4, 1>(a, s);
        launch_down_tiles<W, 3>(a, s);
    }
}

int launch_experts(const duo_moe_config* cfg, const MoeArgs& a, hipStream_t s) {
    if (cfg->scaled) launch_products<Narrow>(a, s);
    else launch_products<Wide>(a, s);
    return duo_internal_hip_ok(hipGetLastError(), "duo_moe_layer");
}

}  // namespace

extern "C" size_t duo_moe_expert_bytes(const duo_moe_config* cfg) { return check_moe(cfg) ? 0 : expert_bytes(cfg); }

extern "C" int duo_moe_pack(const duo_moe_config* cfg, const uint16_t* w_gate, const uint16_t* w_up, const uint16_t* w_down, int expert, void* experts,
                            void* hip_stream) {
    if (const int rc = check_moe(cfg)) return rc;
    if (!w_gate || !w_up || !w_down || !experts) return DUO_ERR_NULL;
    if (expert < 0 || expert >= cfg->n_experts) return DUO_ERR_ARG;
    if (off16(w_gate) || off16(w_up) || off16(w_down) || off16(experts)) return DUO_ERR_ALIGN;
    const int d = cfg->d_model, ff = cfg->d_ff;
    const uint16_t* const src[3] = {w_gate, w_up, w_down};
    char* dst = static_cast<char*>(experts) + (size_t)expert * expert_bytes(cfg);
    for (int i = 0; i < 3; ++i) {
        const int N = i < 2 ? ff : d, K = i < 2 ? d : ff;
        const int rc = cfg->scaled ? duo_scaled_pack(src[i], N, K, dst, hip_stream) : duo_pack_matrix(src[i], N, K, reinterpret_cast<uint16_t*>(dst), hip_stream);
        if (rc) return rc;
        dst += matrix_bytes(cfg, N, K);
    }
    return DUO_OK;
}

extern "C" int duo_moe_workspace_bytes(const duo_moe_config* cfg, int rows, size_t* bytes) {
    if (!bytes) return DUO_ERR_NULL;
    if (const int rc = check_moe(cfg)) return rc;
    if (rows < 1 || rows > DUO_MAX_ROWS) return DUO_ERR_SHAPE;
    *bytes = layout_of(cfg, rows).total;
    return DUO_OK;
}

extern "C" int duo_moe_layer(const duo_moe_config* cfg, const uint16_t* router, const void* experts, const uint16_t* x, int64_t x_stride, int rows,
                             const int32_t* position, uint16_t* y, int64_t y_stride, int32_t* chosen, float* share, void* workspace,
                             size_t workspace_bytes, void* hip_stream) {
    if (const int rc = check_moe(cfg)) return rc;
    if (!router || !experts || !x || !y || !workspace) return DUO_ERR_NULL;
    if (rows < 1 || rows > DUO_MAX_ROWS) return DUO_ERR_SHAPE;
    if (off16(router) || off16(experts) || off16(x) || off16(y) || off16(workspace) || x_stride % 8 || y_stride % 8) return DUO_ERR_ALIGN;
    if (off4(position) || off4(chosen) || off4(share)) return DUO_ERR_ALIGN;
    const int d = cfg->d_model;
    if (rows > 1 && (x_stride < d || y_stride < d || x_stride > DUO_MOE_MAX_STRIDE || y_stride > DUO_MOE_MAX_STRIDE)) return DUO_ERR_SHAPE;
    const MoeLayout lay = layout_of(cfg, rows);
    if (workspace_bytes < lay.total) return DUO_ERR_WORKSPACE;
    char* const ws = static_cast<char*>(workspace);
    MoeArgs a{};
    a.x = x, a.y = y, a.router = router, a.experts = static_cast<const uint8_t*>(experts), a.position = position;
    a.chosen_out = chosen, a.share_out = share;
    a.chosen = reinterpret_cast<int32_t*>(ws + lay.chosen);
    a.share = reinterpret_cast<float*>(ws + lay.share);
    a.logits = reinterpret_cast<double*>(ws + lay.logits);
    a.hidden = reinterpret_cast<u16*>(ws + lay.hidden);
    a.partial = reinterpret_cast<float*>(ws + lay.partial);
    a.x_stride = x_stride, a.y_stride = y_stride;
    a.expert_bytes = expert_bytes(cfg), a.up_at = matrix_bytes(cfg, cfg->d_ff, d), a.down_at = 2 * a.up_at;
    a.rows = rows, a.d = d, a.ff = cfg->d_ff, a.ff_pad = up128(cfg->d_ff), a.n_experts = cfg->n_experts, a.top = cfg->top_k;
    a.renormalise = cfg->renormalise;
    const hipStream_t s = static_cast<hipStream_t>(hip_stream);
    (void)hipGetLastError();  // not of an earlier call
    duo_internal_prof(DUO_PROF_MOE_ROUTER);
    if (router_in_one(a.n_experts, d)) {
        DUO_LAUNCH(moe_router_kernel, dim3((rows + 15) / 16), dim3(64 * ROUTER_WAVES), s, a);
        return launch_experts(cfg, a, s);
    }
    DUO_LAUNCH(moe_logits_kernel, dim3(logit_parts(d), (a.n_experts + 15) / 16, (rows + 15) / 16), dim3(64 * LOGIT_WAVES), s, a);
    duo_internal_prof(DUO_PROF_MOE_ROUTER);
    DUO_LAUNCH(moe_choice_kernel, dim3(rows), dim3(CHOICE_THREADS), s, a);
    return launch_experts(cfg, a, s);
}
