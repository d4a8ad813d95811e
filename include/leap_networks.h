/*
 * leap_networks.h - C ABI of the operators for networks trained through the projector that work on plain arrays: attention over the
 * patches of a volume with learned relative positions, and group norm with an activation, each with its gradients.  (Those on
 * activations in 8 bits are in leap_activations.h.)
 *
 * Conventions (those of leap_activations.h)
 *   - Data pointers are DEVICE pointers owned by the caller, of the current HIP device; nothing is kept, allocated or
 *     freed.  Calls are asynchronous on hip_stream (NULL: the default stream) and can be captured into a graph.
 *   - Strides are distances in elements; the values of a row are neighbours.  No alignment beyond the element's is asked for, but for
 *     workspaces, which begin at a multiple of 16 bytes.
 *   - Outputs are overwritten, have no gaps and must not overlap inputs.  Sums are formed in 32 bits or more, in an order fixed by the
 *     sizes: the same call gives the same bits.
 *   - Every function returns LEAP_OK (0) or a negative status of leap.h; the message is in leap_last_error().
 */
#ifndef LEAP_NETWORKS_H
#define LEAP_NETWORKS_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Attention.  q: [batch][queries][heads][width]; k, v: [batch][keys][kv_heads][width], bfloat16; head h reads the keys and values of head
 * h / (heads / kv_heads).  With x = scale q.k + bias over a query's and a head's keys, p = exp(x) / sum of exp(x) and o = sum of p v; a query
 * without keys has o = 0.
 *
 * The mask, d_mask (NULL: all keys): bytes [batch][keys], items mask_item bytes apart; a key whose byte is 0 is left out, and its k and v
 * do not count whatever they hold.
 *
 * The bias, from d_table [heads][buckets] of table_type (NULL: none): the pair of query i and key j takes the bucket
 * d_bucket_of[d_key_positions[j] - d_query_positions[i] + offsets / 2] of `offsets`; differences beyond either end take that end's, buckets
 * beyond the table's ends its ends'.  Positions (NULL: i and j themselves) are within -2^30 .. 2^30.  Infinities and numbers of any size in the table are fine: -inf
 * leaves a pair out.
 *
 * Sizes: fewer than 2^24 times 128 queries of an item's head, each item's and head's last ones counting as 128; keys alike for the gradients. */
typedef struct {
    int64_t batch, queries, keys, heads, kv_heads, width;
    int64_t q_item, q_row, q_head, k_item, k_row, k_head, v_item, v_row, v_head;       /* strides of an item, of a query or key, of a head */
    int64_t mask_item, offsets, buckets;
    const uint8_t *d_mask;
    const void *d_table;
    const int32_t *d_bucket_of, *d_query_positions, *d_key_positions;
    int32_t table_type;
    float scale;                                                                       /* positive */
} leap_attention_desc;

enum { LEAP_ATTENTION_WIDEST = 128, LEAP_ATTENTION_BUCKETS = 4096 };                   /* the largest width, the most buckets */
enum { LEAP_ATTENTION_OFFSETS = 1 << 24 };                                             /* the most differences; 2^30 for all heads together */

/* o [batch][queries][heads][width] <- attention.  For a backward pass also stats [batch][heads][queries][2] (float: a number m within 8 of the largest exponent of
 * a query's keys, to the base 2, and the sum of 2^(x - m), without a table that sum's logarithm; a query without keys has none of it) and rest [as o] (int16: what has to be added to o's bits, followed by 16 zeros, for those of
 * the 32-bit number that was rounded); NULL: both or neither.  With them the probabilities go into the product with 16 bits instead of 8, with a table with 24.
 * d_work: leap_attention_work() bytes, NULL where that is 0. */
int64_t leap_attention_work(const leap_attention_desc *desc);
int leap_attention(const leap_attention_desc *desc, const void *d_q, const void *d_k, const void *d_v, void *d_o, float *d_stats, void *d_rest,
                   void *d_work, void *hip_stream);

/* Its gradients from that of o: grad [batch][queries][heads][width] with strides; o, stats and rest of the forward pass.  grad_q, grad_k, grad_v: as
 * q, k, v without gaps; grad_table: [heads][buckets], float.  Any of them may be NULL.  Keys that the mask leaves out get zeros; without queries all that is wanted is
 * zeros, and nothing is read.  What is not finite in a query, or in its row of grad, reaches in grad_table the buckets of its pairs alone.
 * A pair's part in grad_table is held to 2^-46 of the largest among those of 128 queries and 64 keys, its sums to 32 bits.
 * d_work: leap_attention_backward_work() bytes (with_table: whether grad_table is wanted), never NULL where there are queries. */
int64_t leap_attention_backward_work(const leap_attention_desc *desc, int32_t with_table);
int leap_attention_backward(const leap_attention_desc *desc, const void *d_grad, int64_t grad_item, int64_t grad_row, int64_t grad_head, const void *d_q,
                            const void *d_k, const void *d_v, const void *d_o, const float *d_stats, const void *d_rest, void *d_grad_q,
                            void *d_grad_k, void *d_grad_v, float *d_grad_table, void *d_work, void *hip_stream);

/* Group norm with an activation, channels last.  x: [items][voxels][channels] of `type`; a group is channels / groups neighbouring channels of an
 * item.  With its mean and rstd = 1 / sqrt(variance + eps) over voxels and channels:  u = (x - mean) * rstd * weight + bias,  y = activation(u).
 * weight, bias: [channels] of weight_type (`type` or float32), or NULL (ones, zeros); y: as x, without gaps.
 * x_item, x_row: distances of items and of voxels.  stats [items][groups][2] (float: mean, rstd) for the backward pass, or NULL.
 * d_work: leap_group_norm_work() bytes, NULL where that is 0.  The sums are formed such that a mean far larger than the deviation costs nothing;
 * a voxel's deviation from the mean is at most 2^55, so that 32 bits hold the sums of their squares, and eight of x have a sum that is finite. */
enum { LEAP_LINEAR = 0, LEAP_RELU = 1, LEAP_SILU = 2 };
int64_t leap_group_norm_work(int64_t items, int64_t voxels, int64_t channels, int64_t groups);
int leap_group_norm(const void *d_x, int32_t type, int64_t x_item, int64_t x_row, const void *d_weight, const void *d_bias, int32_t weight_type, int64_t items,
                    int64_t voxels, int64_t channels, int64_t groups, float eps, int32_t activation, void *d_y, float *d_stats, void *d_work,
                    void *hip_stream);

/* Its gradients from that of y.  x, weight, bias and stats: of the forward pass (x may be what 8 bits held of it).  With du = grad * activation'(u) and
 * h = (x - mean) * rstd:  grad_bias = sum over items and voxels of du,  grad_weight = of du * h,  grad_x = rstd * (du * weight - mean over the group
 * of du * weight - h * mean over the group of du * weight * h).  grad: of `type`, distances grad_item, grad_row.  grad_x: as x, without gaps; grad_weight, grad_bias: [channels]
 * of weight_type; each may be NULL.  The slope of LEAP_RELU at 0 is 0.  d_work: leap_group_norm_backward_work() bytes, 16-byte aligned. */
int64_t leap_group_norm_backward_work(int64_t items, int64_t voxels, int64_t channels, int64_t groups);
int leap_group_norm_backward(const void *d_grad, int64_t grad_item, int64_t grad_row, const void *d_x, int32_t type, int64_t x_item, int64_t x_row,
                             const void *d_weight, const void *d_bias, int32_t weight_type, const float *d_stats, int64_t items, int64_t voxels,
                             int64_t channels, int64_t groups, int32_t activation, void *d_grad_x, void *d_grad_weight, void *d_grad_bias, void *d_work,
                             void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif
