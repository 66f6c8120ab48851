// Which ranges of memory a call over many tensors reads and writes, and whether a written one meets another.  Host code.
#pragma once
#include <stdint.h>

#include <algorithm>
#include <memory>
#include <new>

// Room for `few` ranges on the stack, for more on the heap (ok() tells whether there was any).
template <int FEW>
class FogSpans {
 public:
  explicit FogSpans(int64_t most) {
    if (most > FEW) {
      many_.reset(new (std::nothrow) Span[(size_t)most]);
      spans_ = many_.get();
    }
  }
  bool ok() const { return spans_ != nullptr; }
  void add(const void* p, int64_t bytes, bool written) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    if (p && bytes > 0) spans_[n_++] = {at, at + (uintptr_t)bytes, written};
  }
  // Whether what is written lies apart from everything else.
  bool apart() {
    auto before = [](const Span& a, const Span& b) { return a.begin < b.begin; };
    if (!std::is_sorted(spans_, spans_ + n_, before)) std::sort(spans_, spans_ + n_, before);
    uintptr_t end = 0, written_end = 0;      // of what begins before
    for (int64_t i = 0; i < n_; ++i) {
      if (spans_[i].begin < (spans_[i].written ? end : written_end)) return false;
      end = std::max(end, spans_[i].end);
      if (spans_[i].written) written_end = std::max(written_end, spans_[i].end);
    }
    return true;
  }

 private:
  struct Span { uintptr_t begin, end; bool written; };
  Span few_[FEW];
  std::unique_ptr<Span[]> many_;
  Span* spans_ = few_;
  int64_t n_ = 0;
};
