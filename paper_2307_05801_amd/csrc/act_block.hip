// A feed-forward block as one call, forward and backward: leap_feed_forward8 and its gradient.
//
// The kernels are those of its parts.  What the call saves is the host's time between them, which bounds small blocks: 4096 rows of
// 512 through 1024 hidden values, a training step from Python (du rounded), 258 us operator by operator, 166 as one call each way.
#include "act_common.h"

namespace {

using namespace act;

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

// What the backward pass reads, one array's codes and scales after the other's, each from a multiple of 16 bytes on; or what only the forward
// pass does, the norm's output and the gated rows.
struct kept_block {
    uint8_t *normed, *normed_scales, *sum = nullptr, *sum_scales = nullptr, *gated, *gated_scales, *gate = nullptr, *gate_scales = nullptr;
    float *rstd = nullptr;
    int64_t bytes;
    kept_block(void *base, int64_t rows, int64_t cols, int64_t hidden, bool backward)
    {
        uint8_t *at = (uint8_t *)base;
        const auto take = [&](int64_t n) {
            uint8_t *p = at;
            at += up16(n);
            return p;
        };
        normed = take(rows * cols), normed_scales = take(rows * groups_of(cols));
        if (backward) sum = take(rows * cols), sum_scales = take(rows * groups_of(cols));
        gated = take(rows * hidden), gated_scales = take(rows * groups_of(hidden));
        if (backward) gate = take(rows * 2 * hidden), gate_scales = take(rows * 2 * groups_of(hidden));
        if (backward) rstd = (float *)take(rows * 4);
        bytes = at - (uint8_t *)base;
    }
};

struct block_sizes {
    int64_t rows, cols, hidden, out;
    const void *up, *down;
    int64_t up_stride, down_stride;

    const char *bad() const
    {
        if (const char *why = bad_sizes(rows, cols)) return why;
        if (hidden < 1 || hidden > MOST_COLS / 2) return "hidden columns must be 1 to 2^19";
        if (const char *why = bad_sizes(rows, 2 * hidden)) return why;
        if (const char *why = bad_sizes(rows, out)) return why;
        if (rows > 0x7fffffff) return "more than 2^31 rows";
        if (const char *why = bad_stride(up_stride, 2 * hidden, cols)) return why;
        return bad_stride(down_stride, out, hidden);
    }
    int64_t work(void *kept) const
    {
        const kept_block K(kept, rows, cols, hidden, true);
        const int64_t a = leap_linear8_work(K.normed, rows, cols, up, up_stride, 2 * hidden), b = leap_linear8_work(K.gated, rows, hidden, down, down_stride, out);
        return a > b ? a : b;
    }
    // The parts' workspaces take turns behind du and the norm's gradient (32 bits).
    int64_t dn_bytes() const { return up16(rows * cols * 4); }
    int64_t backward_work(const void *dy, int64_t dy_stride, const du_layout &L) const
    {
        const kept_block K(nullptr, rows, cols, hidden, true);
        int64_t most = leap_rms_norm8_work(rows, cols) * 4;
        for (int64_t n : {leap_linear8_backward_work(dy, dy_stride, K.gated, rows, hidden, down, down_stride, out),
                          leap_linear_gate8_work(dy, dy_stride, down, down_stride, out, rows, hidden),
                          du_backward_work(L, K.normed, rows, cols, up, up_stride, 2 * hidden)})
            most = n > most ? n : most;
        return L.bytes(rows) + dn_bytes() + up16(most);
    }
};

}  // namespace

extern "C" int64_t leap_feed_forward8_kept(int64_t rows, int64_t cols, int64_t hidden)
{
    if (bad_sizes(rows, cols) || hidden < 1 || hidden > MOST_COLS / 2 || bad_sizes(rows, 2 * hidden)) return 0;
    return kept_block(nullptr, rows, cols, hidden, true).bytes;
}

extern "C" int64_t leap_feed_forward8_work(int64_t rows, int64_t cols, const void *d_up, int64_t up_stride, int64_t hidden, const void *d_down,
                                           int64_t down_stride, int64_t out)
{
    const block_sizes S{rows, cols, hidden, out, d_up, d_down, up_stride, down_stride};
    return S.bad() ? 0 : S.work(nullptr);
}

namespace {

int block_forward(const void *d_x, int64_t x_stride, const void *d_residual, int64_t residual_stride, const void *d_norm_weight, int32_t norm_weight_type,
                  float eps, const block_sizes &S, void *d_sum, void *d_y, const kept_block &K, void *d_work, void *hip_stream)
{
    if (!S.up || !S.down || !d_y) return refuse("null data pointer");
    if (norm_weight_type != LEAP_F32 && norm_weight_type != LEAP_BF16) return refuse("the norm's weight must be float32 or bfloat16");
    int rc = leap_rms_norm8(d_x, x_stride, d_residual, residual_stride, LEAP_BF16, d_norm_weight, norm_weight_type, S.rows, S.cols, eps, d_sum, K.normed,
                            K.normed_scales, K.sum, K.sum_scales, K.rstd, hip_stream);
    if (rc == LEAP_OK)
        rc = leap_gated_linear8(K.normed, K.normed_scales, S.rows, S.cols, S.up, S.up_stride, S.hidden, K.gated, K.gated_scales, K.gate, K.gate_scales, d_work,
                                hip_stream);
    if (rc == LEAP_OK) rc = leap_linear8(K.gated, K.gated_scales, S.rows, S.hidden, S.down, S.down_stride, S.out, d_y, d_work, hip_stream);
    return rc;
}

}  // namespace

extern "C" int leap_feed_forward8(const void *d_x, int64_t x_stride, const void *d_residual, int64_t residual_stride, const void *d_norm_weight,
                                  int32_t norm_weight_type, int64_t rows, int64_t cols, float eps, const void *d_up, int64_t up_stride, int64_t hidden,
                                  const void *d_down, int64_t down_stride, int64_t out, void *d_sum, void *d_y, void *d_kept, void *d_work,
                                  void *hip_stream)
{
    const block_sizes S{rows, cols, hidden, out, d_up, d_down, up_stride, down_stride};
    if (const char *why = S.bad()) return refuse(why);
    if (!rows) return LEAP_OK;
    if (unaligned(d_kept)) return refuse("what is kept needs memory from a multiple of 16 bytes on");
    if (unaligned(d_work) && S.work(d_kept)) return refuse(NO_WORK);
    return block_forward(d_x, x_stride, d_residual, residual_stride, d_norm_weight, norm_weight_type, eps, S, d_sum, d_y, kept_block(d_kept, rows, cols, hidden, true),
                         d_work, hip_stream);
}

extern "C" int64_t leap_feed_forward8_alone_work(int64_t rows, int64_t cols, const void *d_up, int64_t up_stride, int64_t hidden, const void *d_down,
                                                 int64_t down_stride, int64_t out)
{
    const block_sizes S{rows, cols, hidden, out, d_up, d_down, up_stride, down_stride};
    return S.bad() ? 0 : kept_block(nullptr, rows, cols, hidden, false).bytes + S.work(nullptr);
}

extern "C" int leap_feed_forward8_alone(const void *d_x, int64_t x_stride, const void *d_residual, int64_t residual_stride, const void *d_norm_weight,
                                        int32_t norm_weight_type, int64_t rows, int64_t cols, float eps, const void *d_up, int64_t up_stride, int64_t hidden,
                                        const void *d_down, int64_t down_stride, int64_t out, void *d_sum, void *d_y, void *d_work, void *hip_stream)
{
    const block_sizes S{rows, cols, hidden, out, d_up, d_down, up_stride, down_stride};
    if (const char *why = S.bad()) return refuse(why);
    if (!rows) return LEAP_OK;
    if (unaligned(d_work)) return refuse(NO_WORK);
    const kept_block K(d_work, rows, cols, hidden, false);
    return block_forward(d_x, x_stride, d_residual, residual_stride, d_norm_weight, norm_weight_type, eps, S, d_sum, d_y, K, (uint8_t *)d_work + K.bytes, hip_stream);
}

namespace {

int64_t block_backward_work(bool fine, const void *d_dy, int64_t dy_stride, const block_sizes &S)
{
    return S.bad() || bad_stride(dy_stride, S.rows, S.out) ? 0 : S.backward_work(d_dy, dy_stride, padded_layout(S.hidden, fine));
}

int block_backward(bool fine, const void *d_dy, int64_t dy_stride, const void *d_grad_sum, int64_t grad_sum_stride, const void *d_norm_weight,
                   int32_t norm_weight_type, const block_sizes &S, const void *d_kept, void *d_grad_x, void *d_grad_norm_weight, void *d_grad_up,
                   void *d_grad_down, void *d_work, void *hip_stream)
{
    if (const char *why = S.bad()) return refuse(why);
    const int64_t rows = S.rows, cols = S.cols, hidden = S.hidden, out = S.out;
    if (const char *why = bad_stride(dy_stride, rows, out)) return refuse(why);
    if (rows && unaligned(d_kept)) return refuse("what is kept needs memory from a multiple of 16 bytes on");
    if (rows && (!d_dy || !S.up || !S.down)) return refuse("null data pointer");
    if (const char *why = d_grad_sum ? bad_stride(grad_sum_stride, rows, cols) : nullptr) return refuse(why);
    if (norm_weight_type != LEAP_F32 && norm_weight_type != LEAP_BF16) return refuse("the norm's weight must be float32 or bfloat16");
    if (rows && (d_grad_x || d_grad_norm_weight) && !d_norm_weight) return refuse("null data pointer");
    if (rows && d_grad_norm_weight && !d_grad_x) return refuse("the norm's weight gradient comes with grad_x");
    if (unaligned(d_work)) return refuse(NO_WORK);
    const kept_block K((void *)d_kept, rows, cols, hidden, true);
    // The matrix units take bfloat16.  A fine du is two of those, and its products take twice as long (262144 x 512 through 1024, forward and backward:
    // 4.79 ms, 3.53); all gradients are 0.0017 of their norm off, their own rounding.  With du rounded, which a caller may ask for, grad_up is 0.0024
    // off and grad_norm_weight 0.0024 to 0.0034.  32 bits between the product and the norm: a rounding less in grad_x.
    const du_layout L = padded_layout(hidden, fine);
    uint8_t *const du = (uint8_t *)d_work, *const dn = du + L.bytes(rows), *const work = dn + S.dn_bytes();
    int rc = LEAP_OK;
    if (d_grad_down)
        rc = leap_linear8_backward(d_dy, dy_stride, K.gated, K.gated_scales, rows, hidden, S.down, S.down_stride, out, nullptr, LEAP_BF16, d_grad_down, work, hip_stream);
    if (rc == LEAP_OK && (d_grad_x || d_grad_up)) {
        rc = linear_gate8_backward(d_dy, dy_stride, S.down, S.down_stride, out, K.gate, K.gate_scales, rows, hidden, du, L, work, hip_stream);
        if (rc == LEAP_OK)
            rc = du_backward(du, L, K.normed, K.normed_scales, rows, cols, S.up, S.up_stride, 2 * hidden, d_grad_x ? dn : nullptr, LEAP_F32, d_grad_up, work,
                             hip_stream);
    }
    if (rc == LEAP_OK && (d_grad_x || d_grad_norm_weight))
        rc = leap_rms_norm8_backward(dn, LEAP_F32, cols, d_grad_sum, grad_sum_stride, LEAP_BF16, K.sum, K.sum_scales, K.rstd, d_norm_weight, norm_weight_type,
                                     rows, cols, d_grad_x, d_grad_norm_weight, (float *)work, hip_stream);
    return rc;
}

}  // namespace

extern "C" int64_t leap_feed_forward8_backward_work(const void *d_dy, int64_t dy_stride, int64_t rows, int64_t cols, const void *d_up, int64_t up_stride,
                                                    int64_t hidden, const void *d_down, int64_t down_stride, int64_t out)
{
    return block_backward_work(false, d_dy, dy_stride, {rows, cols, hidden, out, d_up, d_down, up_stride, down_stride});
}

extern "C" int leap_feed_forward8_backward(const void *d_dy, int64_t dy_stride, const void *d_grad_sum, int64_t grad_sum_stride, const void *d_norm_weight,
                                           int32_t norm_weight_type, int64_t rows, int64_t cols, const void *d_up, int64_t up_stride, int64_t hidden,
                                           const void *d_down, int64_t down_stride, int64_t out, const void *d_kept, void *d_grad_x,
                                           void *d_grad_norm_weight, void *d_grad_up, void *d_grad_down, void *d_work, void *hip_stream)
{
    return block_backward(false, d_dy, dy_stride, d_grad_sum, grad_sum_stride, d_norm_weight, norm_weight_type,
                          {rows, cols, hidden, out, d_up, d_down, up_stride, down_stride}, d_kept, d_grad_x, d_grad_norm_weight, d_grad_up, d_grad_down, d_work, hip_stream);
}

extern "C" int64_t leap_feed_forward8_backward_fine_work(const void *d_dy, int64_t dy_stride, int64_t rows, int64_t cols, const void *d_up, int64_t up_stride,
                                                         int64_t hidden, const void *d_down, int64_t down_stride, int64_t out)
{
    return block_backward_work(true, d_dy, dy_stride, {rows, cols, hidden, out, d_up, d_down, up_stride, down_stride});
}

extern "C" int leap_feed_forward8_backward_fine(const void *d_dy, int64_t dy_stride, const void *d_grad_sum, int64_t grad_sum_stride, const void *d_norm_weight,
                                                int32_t norm_weight_type, int64_t rows, int64_t cols, const void *d_up, int64_t up_stride, int64_t hidden,
                                                const void *d_down, int64_t down_stride, int64_t out, const void *d_kept, void *d_grad_x,
                                                void *d_grad_norm_weight, void *d_grad_up, void *d_grad_down, void *d_work, void *hip_stream)
{
    return block_backward(true, d_dy, dy_stride, d_grad_sum, grad_sum_stride, d_norm_weight, norm_weight_type,
                          {rows, cols, hidden, out, d_up, d_down, up_stride, down_stride}, d_kept, d_grad_x, d_grad_norm_weight, d_grad_up, d_grad_down, d_work, hip_stream);
}
