// Whether buffers of a call share memory (plain host code: tests walk it on the CPU).
#pragma once
#include <stdint.h>

#include <algorithm>

namespace ax {

// `rows` runs of `bytes`, one every `stride` (>= bytes) bytes; a null pointer is no memory
class Region {
 public:
  Region(const void* p, long rows, long stride, long bytes) : first_((uintptr_t)p), rows_(p ? rows : 0), stride_(stride), bytes_(bytes) {
    if (bytes_ <= 0) rows_ = 0;
    if (rows_ > 1 && stride_ == bytes_) {  // one run
      bytes_ = (long)std::min<__int128>((__int128)rows_ * bytes_, INT64_MAX);
      rows_ = 1;
    }
  }
  Region(const void* p, long bytes) : Region(p, 1, bytes, bytes) {}

  bool same(const Region& o) const {
    return first_ == o.first_ && rows_ == o.rows_ && bytes_ == o.bytes_ && (rows_ <= 1 || stride_ == o.stride_);
  }
  // Ranges that lie apart share nothing, nor do runs of one stride that fall between each other, nor does a single run between
  // two others; of different strides none are taken apart.
  bool meets(const Region& o) const {
    if (rows_ <= 0 || o.rows_ <= 0 || end() <= o.first_ || o.end() <= first_) return false;
    const Region &lo = first_ <= o.first_ ? *this : o, &hi = first_ <= o.first_ ? o : *this;
    if (lo.rows_ == 1) return true;  // it reaches the other's first run
    if (hi.rows_ > 1 && hi.stride_ != lo.stride_) return true;
    const uintptr_t d = (hi.first_ - lo.first_) % (uintptr_t)lo.stride_;  // hi starts so far behind one of lo's runs
    return d < (uintptr_t)lo.bytes_ || d + (uintptr_t)hi.bytes_ > (uintptr_t)lo.stride_;
  }

 private:
  uintptr_t end() const {
    const unsigned __int128 e = (unsigned __int128)first_ + (unsigned __int128)(rows_ - 1) * (unsigned __int128)stride_ + (unsigned __int128)bytes_;
    return e > UINTPTR_MAX ? UINTPTR_MAX : (uintptr_t)e;
  }
  uintptr_t first_;
  long rows_, stride_, bytes_;
};

}  // namespace ax
