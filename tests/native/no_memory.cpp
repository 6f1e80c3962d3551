// operator new that fails when it is told to: loaded in front of the library under test.  Test infrastructure.
#include <cstdlib>
#include <new>

namespace {
long left = -1;                                     // allocations until one fails, -1: none does
}

extern "C" {
void new_fails_after(long n) { left = n; }
int new_has_failed() { return left < 0; }
}

void *operator new(size_t n) {
  if (left >= 0 && left-- == 0) throw std::bad_alloc();
  void *p = malloc(n ? n : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
void *operator new[](size_t n) { return operator new(n); }
void operator delete(void *p) noexcept { free(p); }
void operator delete[](void *p) noexcept { free(p); }
void operator delete(void *p, size_t) noexcept { free(p); }
void operator delete[](void *p, size_t) noexcept { free(p); }
