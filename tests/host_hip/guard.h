// Arrays that begin behind, or end before, a page without access.
#pragma once

#include <sys/mman.h>

#include <cstddef>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>

class Guarded {
 public:
  // at_end: the array ends at the page behind it, else it begins at the one before it.
  Guarded(size_t bytes, bool at_end) : bytes_(bytes) {
    const size_t page = 4096, body = (bytes + page - 1) / page * page;
    all_ = body + 2 * page;
    base_ = (char*)mmap(nullptr, all_, PROT_NONE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0);
    if (base_ == MAP_FAILED || (body && mprotect(base_ + page, body, PROT_READ | PROT_WRITE))) {
      std::perror("mmap");
      std::exit(2);
    }
    at_ = base_ + page + (at_end ? body - bytes : 0);
    std::memset(at_, 0xa5, bytes);  // what was there before
  }
  ~Guarded() { munmap(base_, all_); }
  Guarded(const Guarded&) = delete;
  void* get() const { return bytes_ ? at_ : nullptr; }
  template <class T>
  T* as() const {
    return static_cast<T*>(get());
  }

 private:
  char* base_;
  char* at_;
  size_t bytes_, all_;
};
