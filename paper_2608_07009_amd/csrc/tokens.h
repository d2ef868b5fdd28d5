// Token records (hisparse_kv_desc_t): their layout and the host checks shared by the calls that
// write, read and attend to them.
#pragma once

#include "internal.h"

namespace hisparse {

constexpr int kMaxTokenRecordBytes = 8 << 20;

// Where a token's parts lie inside its record.
struct KvLayout {
  int32_t row_bytes;     // from one token's row to the next
  int32_t rope_offset;   // 8-bit latent records: the rotary dims, 128 bytes per token
  int32_t scale_offset;  // 8-bit records: the scales, 8 (grouped) or 4 (latent) bytes per token
  int32_t tpr_shift;
};

inline KvLayout kv_layout(const hisparse_kv_desc_t& d) {
  KvLayout l{};
  while ((1 << l.tpr_shift) < d.tokens_per_record) ++l.tpr_shift;
  const int n = d.tokens_per_record;
  if (d.type == HISPARSE_KV_BF16) {
    l.row_bytes = d.record_bytes / n;
  } else {
    l.row_bytes = d.layout == HISPARSE_KV_GROUPED ? 256 : 512;
    l.rope_offset = n * l.row_bytes;
    l.scale_offset = l.rope_offset + (d.layout == HISPARSE_KV_GROUPED ? 0 : n * 128);
  }
  return l;
}

// Launches on a stream go to the stream's device, whichever is current.
class StreamDevice {
 public:
  explicit StreamDevice(hipStream_t s) {
    hipDevice_t d = 0;
    int cur = 0;
    if (s && hipStreamGetDevice(s, &d) == hipSuccess && hipGetDevice(&cur) == hipSuccess &&
        (int)d != cur && hipSetDevice((int)d) == hipSuccess)
      back_ = cur;
  }
  ~StreamDevice() {
    if (back_ >= 0) (void)hipSetDevice(back_);
  }
  StreamDevice(const StreamDevice&) = delete;
  StreamDevice& operator=(const StreamDevice&) = delete;

 private:
  int back_ = -1;
};

}  // namespace hisparse
