// Host-side declarations of the kernels over dense rows (routing and its choice, products in 8 and 4 bits, embedding, gradient norms).
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/seer.h"

namespace seer {

int hip_fail(hipError_t e);                 // records e for seer_last_hip_error and gives SEER_EHIP

void launch_route(const void *expert, bool wide /* 64-bit entries */, uint32_t count, uint32_t experts, int32_t *expert_ptr,
                  int32_t *slot_choice, int32_t *choice_slot, void *workspace, hipStream_t st);
size_t route_workspace_bytes(uint32_t count, uint32_t experts);

struct RouteRows {                          // passed to the kernels by value
    const int32_t *choice_slot;             // null (launch_quantize): row t goes to row t
    uint32_t tokens, choices, cols;
};
void launch_route_gather(const RouteRows &r, const float *weight, const seer_dense &x, const seer_dense &out, hipStream_t st);
void launch_route_combine(const RouteRows &r, const float *weight, const seer_dense &z, const seer_dense &y, hipStream_t st);
void launch_route_grad(const RouteRows &r, const float *weight, const seer_dense &dy, const seer_dense *z, const seer_dense *dz,
                       float *dweight, hipStream_t st);
void launch_quantize(const RouteRows &r, const seer_dense &x, const seer_dense &q, float *scale, hipStream_t st);

struct I8Args {
    const int8_t *a, *b;
    const float *a_scale, *b_scale;
    const int32_t *group_ptr;               // null: one group of all rows
    void *out;
    int64_t lda, ldb, ldo;
    uint32_t rows, channels, columns, groups;
    int32_t type;
};
struct I8Plan { int32_t kernel /* seer_i8_kernel */; uint32_t tokens /* to a tile */, shares /* of the columns */; };
bool i8_product_fits(const I8Args &a);
I8Plan i8_plan(const I8Args &a);            // by sizes and by where the operands lie
size_t i8_workspace_bytes(uint32_t rows, uint32_t channels, uint32_t columns, uint32_t groups);
void launch_i8_product(const I8Args &a, const I8Plan &p, void *workspace, hipStream_t st);

struct Mx4Args {
    const uint8_t *a, *b, *a_scale, *b_scale;
    const int32_t *group_ptr;               // null: one group of all rows
    void *out;
    int64_t lda, ldb, ldsa, ldsb, ldo;      // bytes, and elements of out
    uint32_t rows, channels, blocks, groups;
    int32_t type;
};
void launch_mx4_quantize(const RouteRows &r, const seer_dense &x, const seer_mx4 &q, hipStream_t st);
bool mx4_product_fits(const Mx4Args &a);
struct Mx4Plan { int32_t kernel /* seer_mx4_kernel */; uint32_t tokens /* to a tile */, shares /* of the columns */; };
Mx4Plan mx4_plan(const Mx4Args &a);         // by sizes and distances of rows
size_t mx4_workspace_bytes(uint32_t rows, uint32_t channels, uint32_t blocks, uint32_t groups);
void launch_mx4_product(const Mx4Args &a, const Mx4Plan &p, void *workspace, hipStream_t st);

constexpr uint32_t kGradParts = 2048;       // partial sums of squares
inline size_t grad_workspace_bytes() { return kGradParts * sizeof(double); }
void launch_grad_norm(const seer_grad *tensors, int32_t count, float *norm, void *workspace, hipStream_t st);
void launch_grad_clip(const seer_grad *tensors, int32_t count, float max_norm, float *norm, void *workspace, hipStream_t st);

void launch_choose(const seer_dense &logits, const float *bias, const seer_choice &how, int32_t *expert, float *weight, hipStream_t st);
void launch_choose_grad(const seer_dense &logits, const seer_choice &how, const int32_t *expert, const float *dweight,
                        const seer_dense &dlogits, hipStream_t st);

void launch_embed(const void *token, bool wide /* 64-bit entries */, uint32_t tokens, const seer_dense &table, float scale,
                  const seer_dense &out, hipStream_t st);
size_t embed_grad_workspace_bytes(uint32_t count, uint32_t rows, uint32_t cols);
void launch_embed_grad(const void *token, bool wide, const seer_dense &dy, float scale, bool accumulate, const seer_dense &dtable,
                       void *workspace, hipStream_t st);

} // namespace seer
