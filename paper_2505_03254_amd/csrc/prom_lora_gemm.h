// The product with the shared ternary weights, adapters added on the way out (prom_lora_gemm.hip).
#pragma once
#include "prom_lora.h"

namespace prom {

// Channels of a row of bf16 planes: whole steps of 64, zeros behind the last channel.
inline int lora_padded(int channels) { return (channels + 63) / 64 * 64; }

// Sorted rows (a.rows).  planes: the input is bf16 planes [m positions][a.planes][a.Kp] instead of int8 [m][K].
void lora_gemm(const LoraGemmArgs &a, int adapter_type, int out_type, bool planes, hipStream_t st);
// rows * rank up to which a few rows' product forms hid itself: a row's adapter passes every workgroup.
constexpr int kFuseMost = 32;
// At most 64 rows in their own order, int8 input.  With a.hid_out (at most kFuseMost numbers) hid is formed on the way from a.first and written there.
void lora_gemm_few(const LoraGemmArgs &a, int adapter_type, int out_type, hipStream_t st);

}  // namespace prom
