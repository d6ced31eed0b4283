// C ABI of the rotation on its own (include/sv_rope.h): argument checks and the launch.
#include "../../include/sv_rope.h"

#include "desc_checks.hpp"
#include "layout_rules.hpp"
#include "rotate.hpp"

namespace {

using namespace sv;

constexpr int64_t kMostHeads = 1 << 24;

bool aligned8(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 7u) == 0; }

// Do x and y describe the same rows?
bool same_rows(const Shape &x, const Shape &y) { return x.st.b == y.st.b && x.st.h == y.st.h && x.st.n == y.st.n; }

}  // namespace

extern "C" sv_status sv_rope3d_rotate(const void *Q, const void *K, const sv_tensor_desc *x, const sv_rope3d *rope, const int32_t *positions,
                                      int inverse, void *YQ, void *YK, const sv_tensor_desc *y, void *stream)
{
    if (!Q || !YQ || !rope || (K == nullptr) != (YK == nullptr)) return SV_ERR_NULL;
    Shape in, out;
    sv_status rc = check_desc(x, &in, false, kMostHeads);
    if (rc != SV_OK) return rc;
    rc = check_desc(y, &out, false, kMostHeads);
    if (rc != SV_OK) return rc;
    if (x->B != y->B || x->H != y->H || x->N != y->N || x->d != y->d || x->dtype != y->dtype) return SV_ERR_SHAPE;
    if (rope->frames <= 0 || rope->rows <= 0 || rope->cols <= 0 || rope->n_t < 0 || rope->n_h < 0 || rope->n_w < 0) return SV_ERR_SHAPE;
    if ((int64_t)rope->n_t + rope->n_h + rope->n_w != in.d / 2) return SV_ERR_SHAPE;
    if (!positions && ((int64_t)rope->frames * rope->rows > in.N || (int64_t)rope->frames * rope->rows * rope->cols != in.N)) return SV_ERR_SHAPE;
    if ((rope->n_t && !rope->cs_t) || (rope->n_h && !rope->cs_h) || (rope->n_w && !rope->cs_w)) return SV_ERR_NULL;
    if (!aligned16(Q) || !aligned16(K) || !aligned16(YQ) || !aligned16(YK)) return SV_ERR_ALIGN;
    if (!aligned8(rope->cs_t) || !aligned8(rope->cs_h) || !aligned8(rope->cs_w) || !aligned4(positions)) return SV_ERR_ALIGN;
    if (((YQ == Q || (K && YK == K)) && !same_rows(in, out)) || YQ == K || YK == Q || YQ == YK) return SV_ERR_SHAPE;

    RotateArgs a{};
    a.x[0] = Q; a.x[1] = K;
    a.y[0] = YQ; a.y[1] = YK;
    a.sx = in.st; a.sy = out.st;
    a.B = in.B; a.H = in.H; a.N = in.N;
    a.tensors = K ? 2 : 1;
    a.frames = rope->frames; a.rows = rope->rows; a.cols = rope->cols;
    a.n_t = rope->n_t; a.n_h = rope->n_h; a.n_w = rope->n_w;
    a.cs_t = rope->cs_t; a.cs_h = rope->cs_h; a.cs_w = rope->cs_w;
    a.positions = positions;
    a.sign = inverse ? -1.f : 1.f;
    a.own_lines = !TokenLayout{out.BH, out.H, out.d, out.elem_bytes, out.st.h, out.st.n}.shares_lines();
    with_head_dim(in.d, [&](auto D) {
        auto go = [&](auto t) {
            using W = RotateShape<decltype(t), D()>;
            const int64_t tiles = ((int64_t)in.N + W::kTokens - 1) / W::kTokens;
            // fewer heads per workgroup until the chip has something to do: 2 048 workgroups (32 760 tokens of 32 heads of 64 93 us with as many,
            // 81 with twice; 4 680 tokens 15 and 19)
            int group = in.H;
            while (group > 1 && tiles * in.B * ((in.H + group - 1) / group) < 2048) group = (group + 1) / 2;
            a.head_group = group;
            const int64_t wgs = tiles * in.B * ((in.H + group - 1) / group);
            if (!grid_ok(wgs, kThreads)) rc = SV_ERR_SHAPE;
            else rotate_rows<decltype(t), D()><<<(unsigned)wgs, kThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
        };
        if (in.bf16) go(uint16_t{});
        else go(float{});
    });
    if (rc != SV_OK) return rc;
    return hipGetLastError() == hipSuccess ? SV_OK : SV_ERR_LAUNCH;
}
