// Host side of the operators without a context for a policy that answers in tokens: argument validation and launches of
// ppo_dropout, ppo_token_logp(_backward), ppo_token_loss, ppo_pair_loss and ppo_token_gae.
#include "../../include/ppo_learner.h"

#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include <algorithm>
#include <type_traits>

#include "dropout.hip.h"
#include "static_error.h"
#include "token_rows.hip.h"
#include "token_seq.hip.h"

namespace {

int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return ppo_static_fail(code, buf);
}

#define LAUNCHCHK(what)                                                                                            \
  do {                                                                                                             \
    hipError_t e_ = hipGetLastError();                                                                             \
    if (e_ != hipSuccess) return fail(PPO_EHIP, "launch of %s failed: %s", what, hipGetErrorString(e_));           \
  } while (0)

constexpr int64_t MAX_ROWS = PPO_TOKEN_MAX_ROWS;      // 256 threads each are a grid of fewer than 2^32; the wider groups belong to rows so
                                                      // long that memory holds too few of them
constexpr int64_t MAX_PAIRS = PPO_TOKEN_MAX_ROWS / 2;
constexpr int64_t MAX_COLS = (int64_t)1 << 30, MAX_STRIDE = (int64_t)1 << 40, MAX_SEQUENCES = (int64_t)1 << 30, MAX_TOKENS = (int64_t)1 << 34;

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool finite_in(double v, double lo, double hi) { return v >= lo && v <= hi; }
bool usable_temperature(float t) { return t > 0 && isfinite(t) && isfinite(2.f / t); }  // log2(e) / t is a factor in the kernels
bool aligned(const void* p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }
int elem_bytes(int32_t dtype) { return dtype == 0 ? 4 : 2; }

// An array of rows: present, aligned to its type, rows that do not overlap.
int check_rows(const char* name, const void* p, int32_t dtype, int64_t cols, int64_t ld) {
  if (!p) return fail(PPO_EINVAL, "%s is NULL", name);
  if (!aligned(p, elem_bytes(dtype))) return fail(PPO_EINVAL, "%s is not aligned to its element type", name);
  if (ld < cols || ld > MAX_STRIDE) return fail(PPO_ESHAPE, "%s: row stride %lld does not hold rows of %lld", name, (long long)ld, (long long)cols);
  return PPO_OK;
}
int check_array(const char* name, const void* p, int bytes, bool needed) {
  if (!p && needed) return fail(PPO_EINVAL, "%s is NULL", name);
  if (p && !aligned(p, bytes)) return fail(PPO_EINVAL, "%s is not aligned to its element type", name);
  return PPO_OK;
}
int check_ws(const void* ws, int64_t have, int64_t want) {
  if (want == 0) return PPO_OK;
  if (!ws) return fail(PPO_EINVAL, "d_ws is NULL");
  if (!aligned(ws, 16)) return fail(PPO_EINVAL, "d_ws is not 16-byte aligned");
  if (have < want) return fail(PPO_EINVAL, "d_ws has %lld bytes, %lld are needed", (long long)have, (long long)want);
  return PPO_OK;
}
#define CHECK(call)        \
  do {                     \
    const int rc_ = (call); \
    if (rc_) return rc_;   \
  } while (0)

int check_sizes(int32_t dtype, int64_t rows, int64_t vocab) {
  if (dtype < 0 || dtype > 2) return fail(PPO_EINVAL, "dtype must be 0 (fp32), 1 (bf16) or 2 (fp16)");
  if (rows < 0 || rows > MAX_ROWS) return fail(PPO_ESHAPE, "rows must be in [0, %lld] (got %lld)", (long long)MAX_ROWS, (long long)rows);
  if (vocab < 1 || vocab > PPO_TOKEN_MAX_VOCAB) return fail(PPO_ESHAPE, "vocab must be in [1, %d] (got %lld)", PPO_TOKEN_MAX_VOCAB, (long long)vocab);
  return PPO_OK;
}

// Rows in slices (k_token_part and what follows it): long rows that would leave part of the chip idle.  One more launch, 2 us, buys
// the other CUs' arithmetic.  us a call in slices and whole (log-probability by blocks of 256 threads), among others:
//   log-probability, bf16   16 x 50000 11 and 8, 16 x 100000 11 and 12, 16 x 128000 10 and 15, 255 x 128000 16 and 19, 400 x 128000 22 and 22
//   loss, bf16              16 x 50000 14 and 12, 16 x 128000 14 and 19, 96 x 100000 16 and 18, 128 x 100000 17 and 19, 200 x 128000 30 and 24
//   loss, fp32              16 x 100000 14 and 16, 64 x 100000 16 and 18, 80 x 100000 20 and 19, 96 x 100000 24 and 20, 80 x 160000 30 and 31
// A call alone, 20 to 30 us, gains from 41000 (loss) and 50000 logits (log-probability) on: 16 x 50000 23 and 25, 20.5 and 20.6.
constexpr int MAX_SLICES = 64, SLICED_ROWS = 255, SLICED_LOSS_ROWS = 96, SLICED_LOSS_ROWS_FP32 = 72;
int slices_of(int64_t rows, int64_t vocab, int64_t most_rows) {
  if (rows > most_rows || vocab <= 40960) return 1;
  return (int)std::min<int64_t>(std::min<int64_t>(cdiv(1024, rows), cdiv(vocab, 4096)), MAX_SLICES);
}
// slices of a multiple of 64 elements, all but the last of one length, none empty
void set_slices(RowArgs& a, int64_t most_rows) {
  const int s = slices_of(a.rows, a.vocab, most_rows);
  a.slice_len = (int32_t)(cdiv(cdiv(a.vocab, s), 64) * 64);
  a.slices = (int32_t)cdiv(a.vocab, a.slice_len);
}

// Workspace of a call on rows: parts of the slices (16 bytes each; enough for any type); for the loss then the rows' records and the sums of
// the blocks that add those up, or nothing where one block does it all.
int64_t parts_bytes(int64_t rows, int64_t vocab, int64_t most_rows) {
  const int s = slices_of(std::max<int64_t>(rows, 1), vocab, most_rows);
  return s > 1 ? rows * s * 16 : 0;
}
bool small_loss(int64_t rows, int64_t vocab) { return rows <= SMALL_ROWS && vocab <= SMALL_VOCAB && rows * vocab <= SMALL_LOGITS; }
int stats_blocks(int64_t rows) { return (int)std::max<int64_t>(1, std::min<int64_t>(cdiv(rows, STATS_ROWS), 1024)); }
int64_t stats_offset(int64_t rows, int64_t vocab) {
  return (parts_bytes(rows, vocab, SLICED_LOSS_ROWS) + rows * (int64_t)sizeof(LossRecord) + 15) / 16 * 16;
}

// f(element type) for the type named by dtype
template <class F>
void with_type(int32_t dtype, F f) {
  if (dtype == 0) f(float());
  else if (dtype == 1) f(bf16_t());
  else f(f16_t());
}

// Groups of threads per sequence of the preference loss: enough that few long sequences fill the chip, none with less than 1024 tokens
// on the average.
int pair_slices(int64_t pairs, int64_t tokens) {
  if (pairs == 0) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>({cdiv(2048, 2 * pairs), tokens / (2 * pairs) / 1024, 256}));
}

int64_t gae_tiles(int64_t tokens) { return cdiv(tokens, GAE_TILE); }

template <class F>
void with_flag(bool on, F f) {
  if (on) f(std::true_type());
  else f(std::false_type());
}

// The kernel of a loss: the narrowest group whose registers hold the row; four rows a wave (16 threads each) are 131072 rows of 257 in
// 39 us where one is 86, but fewer and longer chains for few rows (448 of 256: 4.9 and 3.4 us).
template <class T, bool ENT>
void launch_loss(const RowArgs& a, hipStream_t st) {
  const int64_t pieces = cdiv(a.vocab, Piece<T>::N);
  if (a.slices > 1) {
    hipLaunchKernelGGL((k_token_part<T, ENT>), dim3(a.slices, (uint32_t)a.rows), dim3(256), 0, st, a);
    hipLaunchKernelGGL((k_token_loss_slice<T, ENT>), dim3(a.slices, (uint32_t)a.rows), dim3(256), 0, st, a);
    return;
  }
#define LOSS(G, K)                                                                                                                            \
  if (pieces <= G * K) {                                                                                                                      \
    hipLaunchKernelGGL((k_token_loss<T, G, K, ENT>), dim3((uint32_t)cdiv(a.rows, G < 256 ? 256 / G : 1)), dim3(G < 256 ? 256 : G), 0, st, a); \
    return;                                                                                                                                   \
  }
  LOSS(16, 2)
  if (a.rows < 4096) {
    LOSS(64, 1)
    LOSS(64, 2)
  }
  LOSS(16, 4)
  LOSS(16, 8)
  LOSS(64, 4)
  LOSS(64, 8)
  LOSS(256, 4)
  LOSS(256, 8)
  LOSS(256, 16)
  LOSS(512, 16)
  LOSS(1024, 16)
  LOSS(1024, 25)
#undef LOSS
  hipLaunchKernelGGL((k_token_loss_long<T, ENT>), dim3((uint32_t)a.rows), dim3(1024), 0, st, a);
}

}  // namespace

extern "C" {

int ppo_dropout(int32_t dtype, int64_t rows, int64_t cols, const void* d_x, int64_t ld_x, const int64_t* d_row_ids, const void* d_residual,
                int64_t ld_residual, double p, uint64_t seed, uint64_t layer, void* d_y, int64_t ld_y, void* hip_stream) {
  if (dtype < 0 || dtype > 2) return fail(PPO_EINVAL, "dtype must be 0 (fp32), 1 (bf16) or 2 (fp16)");
  if (rows < 0 || rows > MAX_ROWS) return fail(PPO_ESHAPE, "rows must be in [0, %lld] (got %lld)", (long long)MAX_ROWS, (long long)rows);
  if (cols < 0 || cols > MAX_COLS) return fail(PPO_ESHAPE, "columns must be in [0, %lld] (got %lld)", (long long)MAX_COLS, (long long)cols);
  if (!finite_in(p, 0, 1)) return fail(PPO_EINVAL, "p must be in [0, 1]");
  if (rows == 0 || cols == 0) return PPO_OK;
  CHECK(check_rows("d_x", d_x, dtype, cols, ld_x));
  CHECK(check_rows("d_y", d_y, dtype, cols, ld_y));
  if (d_residual) CHECK(check_rows("d_residual", d_residual, dtype, cols, ld_residual));
  CHECK(check_array("d_row_ids", d_row_ids, 8, false));
  const uint32_t border = (uint32_t)(p * 65536 + 0.5);
  const uint64_t G64 = 0x9E3779B97F4A7C15ULL;
  const uint64_t prefix = sm64_mix(sm64_mix(seed + G64) ^ (layer + G64));   // the first two steps of perm_stream
  const DropoutArgs a = {rows, cols, ld_x, ld_residual, ld_y, d_x, d_residual, d_y, d_row_ids, prefix, border,
                         border < 65536 ? 65536.f / (float)(65536 - border) : 0.f};
  hipStream_t st = (hipStream_t)hip_stream;
  with_type(dtype, [&](auto t) {
    with_flag(d_residual != nullptr, [&](auto res) {
      using T = decltype(t);
      constexpr bool RES = decltype(res)::value;
      const int64_t pieces = cdiv(cols, Piece<T>::N);
      if (pieces <= 16 * DROP_PIECES) hipLaunchKernelGGL((k_dropout<T, 16, RES>), dim3((uint32_t)cdiv(rows, 16)), dim3(256), 0, st, a);
      else if (pieces <= 64 * DROP_PIECES) hipLaunchKernelGGL((k_dropout<T, 64, RES>), dim3((uint32_t)cdiv(rows, 4)), dim3(256), 0, st, a);
      else hipLaunchKernelGGL((k_dropout<T, 256, RES>), dim3((uint32_t)cdiv(pieces, 256 * DROP_PIECES), (uint32_t)std::min<int64_t>(rows, 65535), (uint32_t)cdiv(rows, 65535)),
                              dim3(256), 0, st, a);
    });
  });
  LAUNCHCHK("k_dropout");
  return PPO_OK;
}

int64_t ppo_token_logp_ws_bytes(int64_t rows, int64_t vocab) {
  if (rows < 0 || rows > MAX_ROWS || vocab < 1 || vocab > PPO_TOKEN_MAX_VOCAB) return PPO_ESHAPE;
  return parts_bytes(rows, vocab, SLICED_ROWS);
}

int64_t ppo_token_loss_ws_bytes(int64_t rows, int64_t vocab) {
  if (rows < 0 || rows > MAX_ROWS || vocab < 1 || vocab > PPO_TOKEN_MAX_VOCAB) return PPO_ESHAPE;
  if (small_loss(rows, vocab)) return 0;
  return stats_offset(rows, vocab) + (stats_blocks(rows) > 1 ? stats_blocks(rows) * 48 : 0);
}

int ppo_token_logp(int32_t dtype, int64_t rows, int64_t vocab, const void* d_logits, int64_t ld, const int32_t* d_target, float temperature, float* d_logp,
                   float* d_entropy, float* d_stat, void* d_ws, int64_t ws_bytes, void* hip_stream) {
  CHECK(check_sizes(dtype, rows, vocab));
  if (!usable_temperature(temperature)) return fail(PPO_EINVAL, "temperature must be finite and > 0, and so must 2 / temperature");
  if (rows == 0) return PPO_OK;
  CHECK(check_rows("d_logits", d_logits, dtype, vocab, ld));
  CHECK(check_array("d_target", d_target, 4, true));
  CHECK(check_array("d_logp", d_logp, 4, true));
  CHECK(check_array("d_entropy", d_entropy, 4, false));
  CHECK(check_array("d_stat", d_stat, 4, false));
  CHECK(check_ws(d_ws, ws_bytes, ppo_token_logp_ws_bytes(rows, vocab)));
  RowArgs a = {};
  a.rows = rows; a.ld = ld; a.vocab = (int32_t)vocab; a.logits = d_logits; a.target = d_target; a.inv_t = 1.f / temperature;
  a.logp = d_logp; a.entropy = d_entropy; a.stat = d_stat;
  a.part = (float*)d_ws;
  set_slices(a, SLICED_ROWS);
  hipStream_t st = (hipStream_t)hip_stream;
  with_type(dtype, [&](auto t) {
    with_flag(d_entropy != nullptr, [&](auto ent) {
      using T = decltype(t);
      constexpr bool ENT = decltype(ent)::value;
      const int64_t pieces = cdiv(vocab, Piece<T>::N);
      if (a.slices > 1) {
        hipLaunchKernelGGL((k_token_part<T, ENT>), dim3(a.slices, (uint32_t)rows), dim3(256), 0, st, a);
        hipLaunchKernelGGL(k_token_join<ENT>, dim3((uint32_t)cdiv(rows, 4)), dim3(256), 0, st, a);
      } else if (pieces <= 128) hipLaunchKernelGGL((k_token_logp<T, 16, ENT>), dim3((uint32_t)cdiv(rows, 16)), dim3(256), 0, st, a);
      else if (pieces <= 512) hipLaunchKernelGGL((k_token_logp<T, 64, ENT>), dim3((uint32_t)cdiv(rows, 4)), dim3(256), 0, st, a);
      else hipLaunchKernelGGL((k_token_logp<T, 256, ENT>), dim3((uint32_t)rows), dim3(256), 0, st, a);
    });
  });
  LAUNCHCHK("k_token_logp");
  return PPO_OK;
}

int ppo_token_logp_backward(int32_t dtype, int64_t rows, int64_t vocab, const void* d_logits, int64_t ld, const int32_t* d_target, float temperature,
                            const float* d_stat, const float* d_dlogp, const float* d_entropy, const float* d_dentropy, void* d_dlogits, int64_t ld_d,
                            void* hip_stream) {
  CHECK(check_sizes(dtype, rows, vocab));
  if (!usable_temperature(temperature)) return fail(PPO_EINVAL, "temperature must be finite and > 0, and so must 2 / temperature");
  if (rows == 0) return PPO_OK;
  CHECK(check_rows("d_logits", d_logits, dtype, vocab, ld));
  CHECK(check_rows("d_dlogits", d_dlogits, dtype, vocab, ld_d));
  CHECK(check_array("d_target", d_target, 4, true));
  CHECK(check_array("d_stat", d_stat, 4, true));
  CHECK(check_array("d_dlogp", d_dlogp, 4, true));
  CHECK(check_array("d_dentropy", d_dentropy, 4, false));
  CHECK(check_array("d_entropy", d_entropy, 4, d_dentropy != nullptr));
  RowArgs a = {};
  a.rows = rows; a.ld = ld; a.ldd = ld_d; a.vocab = (int32_t)vocab; a.logits = d_logits; a.target = d_target; a.inv_t = 1.f / temperature;
  a.stat = (float*)d_stat; a.dlogp = d_dlogp; a.entropy = (float*)d_entropy; a.dentropy = d_dentropy; a.dlogits = d_dlogits;
  hipStream_t st = (hipStream_t)hip_stream;
  with_type(dtype, [&](auto t) {
    with_flag(d_dentropy != nullptr, [&](auto ent) {
      using T = decltype(t);
      constexpr bool ENT = decltype(ent)::value;
      const int64_t pieces = cdiv(vocab, Piece<T>::N);
      with_flag(rows * vocab * (int64_t)sizeof(T) > PAST_BYTES, [&](auto past) {
        constexpr bool PAST = decltype(past)::value;
        if (pieces <= 16 * BACK_PIECES) hipLaunchKernelGGL((k_token_logp_backward<T, 16, ENT, PAST>), dim3((uint32_t)cdiv(rows, 16)), dim3(256), 0, st, a);
        else if (pieces <= 64 * BACK_PIECES) hipLaunchKernelGGL((k_token_logp_backward<T, 64, ENT, PAST>), dim3((uint32_t)cdiv(rows, 4)), dim3(256), 0, st, a);
        else hipLaunchKernelGGL((k_token_logp_backward<T, 256, ENT, PAST>), dim3((uint32_t)cdiv(pieces, 256 * BACK_PIECES), (uint32_t)std::min<int64_t>(rows, 65535), (uint32_t)cdiv(rows, 65535)),
                                dim3(256), 0, st, a);
      });
    });
  });
  LAUNCHCHK("k_token_logp_backward");
  return PPO_OK;
}

int ppo_token_loss(int32_t dtype, int64_t rows, int64_t vocab, const void* d_logits, int64_t ld, const int32_t* d_target, const float* d_logp_old,
                   const float* d_logp_ref, const float* d_adv, const float* d_weight, const ppo_token_hparams* hp, void* d_dlogits, int64_t ld_d,
                   float* d_logp, float* d_stats, void* d_ws, int64_t ws_bytes, void* hip_stream) {
  CHECK(check_sizes(dtype, rows, vocab));
  if (!hp) return fail(PPO_EINVAL, "hp is NULL");
  if (!usable_temperature(hp->temperature)) return fail(PPO_EINVAL, "temperature must be finite and > 0, and so must 2 / temperature");
  if (!finite_in(hp->clip_lo, 0, 1) || !(hp->clip_hi >= 0) || !isfinite(hp->clip_hi)) return fail(PPO_EINVAL, "clip_lo must be in [0, 1] and clip_hi finite and >= 0");
  if (!(hp->kl_coef >= 0) || !isfinite(hp->kl_coef)) return fail(PPO_EINVAL, "kl_coef must be finite and >= 0");
  if (hp->kl_coef > 0 && rows > 0 && !d_logp_ref) return fail(PPO_EINVAL, "kl_coef > 0 needs d_logp_ref");
  if (!isfinite(hp->ent_coef) || !isfinite(hp->scale) || !isfinite(hp->ent_coef * hp->scale)) return fail(PPO_EINVAL, "ent_coef, scale and their product must be finite");
  CHECK(check_array("d_stats", d_stats, 4, true));
  if (rows > 0) {
    CHECK(check_rows("d_logits", d_logits, dtype, vocab, ld));
    CHECK(check_rows("d_dlogits", d_dlogits, dtype, vocab, ld_d));
    CHECK(check_array("d_target", d_target, 4, true));
    CHECK(check_array("d_logp_old", d_logp_old, 4, true));
    CHECK(check_array("d_logp_ref", d_logp_ref, 4, false));
    CHECK(check_array("d_adv", d_adv, 4, true));
    CHECK(check_array("d_weight", d_weight, 4, false));
    CHECK(check_array("d_logp", d_logp, 4, false));
    CHECK(check_ws(d_ws, ws_bytes, ppo_token_loss_ws_bytes(rows, vocab)));
  }
  RowArgs a = {};
  a.rows = rows; a.ld = ld; a.ldd = ld_d; a.vocab = (int32_t)vocab; a.logits = d_logits; a.target = d_target; a.inv_t = 1.f / hp->temperature;
  a.logp = d_logp; a.dlogits = d_dlogits; a.logp_old = d_logp_old; a.logp_ref = d_logp_ref; a.adv = d_adv; a.weight = d_weight;
  a.clip_lo = hp->clip_lo; a.clip_hi = hp->clip_hi; a.kl_coef = hp->kl_coef; a.ent_coef = hp->ent_coef; a.scale = hp->scale;
  hipStream_t st = (hipStream_t)hip_stream;
  if (small_loss(rows, vocab)) {
    with_type(dtype, [&](auto t) {
      with_flag(hp->ent_coef != 0.f, [&](auto ent) {
        using T = decltype(t);
        constexpr bool ENT = decltype(ent)::value;
        constexpr int HOLDS = 16 * 4 * Piece<T>::N;   // logits that 16 threads hold in four pieces each
        if constexpr (HOLDS < SMALL_VOCAB) {
          if (vocab > HOLDS) {
            hipLaunchKernelGGL((k_token_loss_small<T, 8, ENT>), dim3(1), dim3(1024), 0, st, a, d_stats);
            return;
          }
        }
        hipLaunchKernelGGL((k_token_loss_small<T, 4, ENT>), dim3(1), dim3(1024), 0, st, a, d_stats);
      });
    });
    LAUNCHCHK("k_token_loss_small");
    return PPO_OK;
  }
  if (rows > 0) {
    set_slices(a, dtype == 0 ? SLICED_LOSS_ROWS_FP32 : SLICED_LOSS_ROWS);
    a.part = (float*)d_ws;
    a.record = (float*)d_ws + (a.slices > 1 ? rows * a.slices * 4 : 0);
    with_type(dtype, [&](auto t) {
      with_flag(hp->ent_coef != 0.f, [&](auto ent) { launch_loss<decltype(t), decltype(ent)::value>(a, st); });
    });
    LAUNCHCHK("k_token_loss");
  }
  const int blocks = stats_blocks(rows);
  double* part = (double*)((char*)d_ws + stats_offset(rows, vocab));
  hipLaunchKernelGGL(k_token_stats, dim3(blocks), dim3(1024), 0, st, rows, cdiv(std::max<int64_t>(rows, 1), blocks), (const LossRecord*)a.record, hp->kl_coef, hp->ent_coef, d_stats, part);
  if (blocks > 1) hipLaunchKernelGGL(k_token_stats_join, dim3(1), dim3(1024), 0, st, blocks, hp->kl_coef, hp->ent_coef, d_stats, (const double*)part);
  LAUNCHCHK("k_token_stats");
  return PPO_OK;
}

int64_t ppo_pair_ws_bytes(int64_t pairs, int64_t tokens) {
  if (pairs < 0 || pairs > MAX_PAIRS || tokens < 0 || tokens > MAX_TOKENS) return PPO_ESHAPE;
  return pairs * (int64_t)sizeof(PairRecord) + 2 * pairs * pair_slices(pairs, tokens) * (int64_t)sizeof(double2) + (stats_blocks(pairs) > 1 ? stats_blocks(pairs) * 48 : 0);
}

int ppo_pair_loss(int64_t pairs, int64_t tokens, const float* d_logp, const float* d_logp_ref, const uint8_t* d_mask, const int64_t* d_offsets,
                  const ppo_pair_hparams* hp, float* d_dlogp, float* d_margin, float* d_stats, void* d_ws, int64_t ws_bytes, void* hip_stream) {
  if (pairs < 0 || pairs > MAX_PAIRS || tokens < 0 || tokens > MAX_TOKENS) return fail(PPO_ESHAPE, "pairs or tokens out of range");
  if (!hp) return fail(PPO_EINVAL, "hp is NULL");
  if (hp->kind < 0 || hp->kind > 1) return fail(PPO_EINVAL, "kind must be 0 (sigmoid) or 1 (squared)");
  if (!(hp->beta > 0) || !isfinite(hp->beta)) return fail(PPO_EINVAL, "beta must be finite and > 0");
  if (!finite_in(hp->label_smoothing, 0, 1)) return fail(PPO_EINVAL, "label_smoothing must be in [0, 1]");
  if (!isfinite(hp->scale)) return fail(PPO_EINVAL, "scale must be finite");
  CHECK(check_array("d_stats", d_stats, 4, true));
  CHECK(check_array("d_logp", d_logp, 4, tokens > 0));
  CHECK(check_array("d_logp_ref", d_logp_ref, 4, false));
  CHECK(check_array("d_dlogp", d_dlogp, 4, tokens > 0));
  CHECK(check_array("d_margin", d_margin, 4, false));
  CHECK(check_array("d_offsets", d_offsets, 8, pairs > 0 || tokens > 0));
  CHECK(check_ws(d_ws, ws_bytes, ppo_pair_ws_bytes(pairs, tokens)));
  const PairArgs a = {pairs, tokens, d_logp, d_logp_ref, d_mask, d_offsets, hp->kind, hp->length_mean, hp->beta, hp->label_smoothing, hp->scale,
                      d_dlogp, d_margin, pairs > PAIRS_INLINE ? (PairRecord*)d_ws : nullptr, d_stats};
  hipStream_t st = (hipStream_t)hip_stream;
  const PairGrid g = {pair_slices(pairs, tokens), (double2*)((PairRecord*)d_ws + pairs)};
  const int64_t items = 2 * pairs * g.slices;
  const uint32_t extra = a.record ? 0 : 1;   // the block of the statistics
  const int64_t mean = pairs > 0 ? tokens / (2 * pairs) : 0;
  if (pairs >= 2048 && mean <= 64) {
    hipLaunchKernelGGL(k_pair_sums<16>, dim3((uint32_t)cdiv(items, 16)), dim3(256), 0, st, a, g);
    hipLaunchKernelGGL(k_pair_loss<16>, dim3((uint32_t)cdiv(items, 16) + extra), dim3(256), 0, st, a, g);
  } else if (pairs >= 2048 && mean <= 512) {
    hipLaunchKernelGGL(k_pair_sums<64>, dim3((uint32_t)cdiv(items, 4)), dim3(256), 0, st, a, g);
    hipLaunchKernelGGL(k_pair_loss<64>, dim3((uint32_t)cdiv(items, 4) + extra), dim3(256), 0, st, a, g);
  } else {
    if (pairs > 0) hipLaunchKernelGGL(k_pair_sums<256>, dim3((uint32_t)items), dim3(256), 0, st, a, g);
    const int64_t blocks = pairs > 0 ? items : std::min<int64_t>(cdiv(tokens, 256), 1024);   // no pairs: the gradient is zeros
    hipLaunchKernelGGL(k_pair_loss<256>, dim3((uint32_t)blocks + extra), dim3(256), 0, st, a, g);
  }
  if (a.record) {
    const int blocks = stats_blocks(pairs);
    double* part = (double*)(g.part + items);
    hipLaunchKernelGGL(k_pair_stats, dim3(blocks), dim3(1024), 0, st, pairs, cdiv(pairs, blocks), (const PairRecord*)a.record, hp->scale, d_stats, part);
    if (blocks > 1) hipLaunchKernelGGL(k_pair_stats_join, dim3(1), dim3(1024), 0, st, blocks, hp->scale, d_stats, (const double*)part);
  }
  LAUNCHCHK("the kernels of ppo_pair_loss");
  return PPO_OK;
}

int64_t ppo_token_gae_ws_bytes(int64_t sequences, int64_t tokens) {
  if (sequences < 0 || sequences > MAX_SEQUENCES || tokens < 0 || tokens > MAX_TOKENS) return PPO_ESHAPE;
  const int64_t tiles = gae_tiles(tokens);
  return tiles <= 1 ? 0 : tiles * (int64_t)sizeof(GaeMap) + (tiles > GAE_DIRECT ? tiles * (int64_t)sizeof(double2) : 0);
}

int ppo_token_gae(int64_t sequences, int64_t tokens, const float* d_reward, const float* d_value, const uint8_t* d_mask, const int64_t* d_offsets,
                  const float* d_last_value, double gamma, double lambda, float* d_adv, float* d_ret, void* d_ws, int64_t ws_bytes, void* hip_stream) {
  if (sequences < 0 || sequences > MAX_SEQUENCES || tokens < 0 || tokens > MAX_TOKENS) return fail(PPO_ESHAPE, "sequences or tokens out of range");
  if (!finite_in(gamma, 0, 1) || !finite_in(lambda, 0, 1)) return fail(PPO_EINVAL, "gamma and lambda must be in [0, 1]");
  if (tokens == 0) return PPO_OK;
  CHECK(check_array("d_reward", d_reward, 4, true));
  CHECK(check_array("d_value", d_value, 4, true));
  CHECK(check_array("d_offsets", d_offsets, 8, true));
  CHECK(check_array("d_last_value", d_last_value, 4, false));
  CHECK(check_array("d_adv", d_adv, 4, true));
  CHECK(check_array("d_ret", d_ret, 4, true));
  CHECK(check_ws(d_ws, ws_bytes, ppo_token_gae_ws_bytes(sequences, tokens)));
  const int64_t tiles = gae_tiles(tokens);
  GaeMap* map = tiles > 1 ? (GaeMap*)d_ws : nullptr;
  double2* in = tiles > GAE_DIRECT ? (double2*)d_ws : nullptr;
  if (in) map = (GaeMap*)(in + tiles);
  const GaeArgs a = {sequences, tokens, d_reward, d_value, d_last_value, d_mask, d_offsets, gamma, lambda, d_adv, d_ret, tiles, map, in};
  hipStream_t st = (hipStream_t)hip_stream;
  if (tiles > 1) hipLaunchKernelGGL(k_gae_part, dim3((uint32_t)tiles), dim3(256), 0, st, a);
  if (in) hipLaunchKernelGGL(k_gae_tiles, dim3(1), dim3(1024), 0, st, a);
  hipLaunchKernelGGL(k_token_gae, dim3((uint32_t)tiles), dim3(256), 0, st, a);
  LAUNCHCHK("the kernels of ppo_token_gae");
  return PPO_OK;
}

}  // extern "C"
