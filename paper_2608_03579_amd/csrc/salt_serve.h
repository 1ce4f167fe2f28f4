// Internal declarations of the operators around the apply (salt_serve.cpp and its
// kernels): what they take from a context, and the arguments of their launches.
// Not part of the public ABI (include/salt.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "salt.h"

namespace salt {

// ---- a context, as salt_serve.cpp sees it (salt_runtime.cpp) --------------------
struct CtxView {
  int device, n_cu;
  int bf16;                 // context dtype: 1 bf16, 0 fp32
  int max_tokens;
  int n_tables;
  const salt_shape* tables;
};
// SALT_OK, or why the context takes no call (null, poisoned).
salt_status ctx_live(salt_ctx* c);
CtxView ctx_view(const salt_ctx* c);
// Keep a message and return `s`; poison the context over a failed HIP call.
salt_status ctx_fail(salt_ctx* c, salt_status s, const char* fmt, ...);
salt_status ctx_hip_fail(salt_ctx* c, hipError_t e, const char* what);
// Objects that salt_destroy frees with the context, by address.
typedef void (*OwnedFree)(void*);
bool ctx_own(salt_ctx* c, void* obj, OwnedFree f);
bool ctx_owns(const salt_ctx* c, const void* obj);
bool ctx_disown(salt_ctx* c, void* obj);   // false: not this context's
// The base weights of the context (one object, made by the first salt_pin_base).
void*& ctx_base(salt_ctx* c);

// ---- base weights in 8 bits -------------------------------------------------------
// Codes of W^T in operand order: a tile holds 16 outputs x 128 inputs in 2 KB, tiles
// [out_pad / 16][in blocks].  Lane l of a wave brings output row (l & 15) and, of the
// 128 inputs, 32 (l >> 4) .. + 31 as two 16-byte halves; half h of lane l stands at
// h * 1024 + l * 16, so every wave access is 1 KB in a row, from memory and from LDS
// alike.  Two tiles share 32 outputs: row 4 g + i of tile 2 p is output 32 p + 8 g + i,
// that of tile 2 p + 1 is 32 p + 8 g + 4 + i, so a lane's products (rows 4 g ..
// 4 g + 3) of a tile pair are 8 outputs in a row.  Quantised x: the same, with
// tokens for outputs and row r of tile t for token 16 t + r.
constexpr int kBaseBlock = 128;          // inputs and outputs that share a scale
constexpr int kBaseTile = 2048;          // bytes of a tile
constexpr int kBasePad = 256;            // outputs and tokens are padded to whole product tiles
constexpr int kBaseTables = 16;          // tables of one launch
struct BaseTable {
  uint8_t* w;               // [out_pad / 16][kb][kBaseTile]
  float* sw;                // [kb][out_pad / 128]
  void* y;                  // [T][out]
  int32_t out, n_blk;       // n_blk: out_pad / 128
  int32_t first;            // the launch's work items of earlier tables
};
struct BaseArgs {
  BaseTable tab[kBaseTables];
  const void* x;            // [T][in]
  uint8_t* xq;              // [T_pad / 16][kb][kBaseTile]
  float* sx;                // [kb][T_pad]
  int32_t n_tables, T, T_pad, in, kb;
};
struct BasePinArgs {        // one table's weights in or out
  void* w;                  // [in][ld] context dtype (quantised from, or read back to)
  const uint8_t* q;         // [out][ld] codes and
  const float* sq;          // [out / 128][in / 128] scales that came quantised
  int64_t ld;
  BaseTable tab;
  int32_t in, kb;
};
hipError_t launch_base_pin(const BasePinArgs& a, int bf16, hipStream_t s);      // w -> tab
hipError_t launch_base_pin_codes(const BasePinArgs& a, hipStream_t s);          // q, sq -> tab
hipError_t launch_base_read(const BasePinArgs& a, int bf16, hipStream_t s);     // tab -> w
hipError_t launch_base_product(const BaseArgs& a, int bf16, int n_cu, hipStream_t s);

// ---- the KV cache -------------------------------------------------------------------
// One layer of the pool.  Codes [pages][kv heads][page tokens][head_dim] of k and of v,
// scales [pages][kv heads][page tokens] fp32.  A vector of head_dim values that holds
// one that is not finite has codes 0 and the scale NaN, and a v like that gives its
// k the scale NaN too.
enum KvFormat { kKvE4m3 = 0, kKvInt8 = 1 };
struct KvLayer {
  uint8_t *k, *v;
  float *ks, *vs;
  int32_t kv_heads, dim, log2_page, format;
  float* weight;            // marks, laid out as the scales (null: not tracked): gathered attention weight, and
  int32_t* place;           // position of the token
};
struct KvWriteArgs {
  KvLayer kv;
  const void *k, *v;        // [T][ld], kv head h at h * dim
  int64_t ldk, ldv;         // elements
  const int32_t* slot;      // [T]: page * page tokens + place, or -1
  const int32_t* place;     // [T]: place in the sequence, where the tokens' marks start; null: marks stay as they are
  int32_t T;
};
struct KvReadArgs {
  KvLayer kv;
  void *k, *v;              // [rows][ld]
  int64_t ldk, ldv;
  const int32_t* slot;      // "new": as above, n = T; slots of -1 read as zeros
  const int32_t *page, *row, *count;   // "own": n page references, their first row and tokens
  int32_t n;
};
hipError_t launch_kv_write(const KvWriteArgs& a, int bf16, hipStream_t s);
hipError_t launch_kv_read(const KvReadArgs& a, int bf16, hipStream_t s);

// ---- attention over it ----------------------------------------------------------------
struct AttItem;
struct AttJoin;
struct AttArgs {
  KvLayer kv;
  const void* q;            // [T][ldq], query head h at h * dim
  void* out;                // [T][ldo]
  int64_t ldq, ldo;
  const int32_t* pages;     // page of each reference
  const int32_t* order;     // token order of the items
  const AttItem* items;
  const AttJoin* joins;
  float* part;              // [rows][dim] weighted sums of v, and
  float* stat;              // [rows][2] max (log2) and sum, of rows in pieces
  int32_t heads, group;     // query heads, and those of one kv head
  int32_t n_kind[4];        // items of each kind; kinds 2, 1, 0 (a block each), then 3 (a wave each)
  int32_t n_joins;
  float scale;              // of the logits
};
hipError_t launch_attend(const AttArgs& a, int bf16, hipStream_t s);

}  // namespace salt
