// Loads from memory straight into LDS, and the waits that go with them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cd {

// 16 bytes per lane from a buffer straight into LDS: lane l of the wave writes its vector at
// lds_addr + 16*l (lds_addr is uniform over the wave and travels in M0); an offset at or beyond the buffer's size
// writes zeros, so that a masked-out vector costs one select instead of a branch around the load.  The compiler does
// not see these loads: the kernel waits for them itself (wait_vmem) before a barrier publishes the tile.
typedef int rsrc_words_t __attribute__((ext_vector_type(4)));
// the four descriptor words of a raw buffer (stride 0): base address, size in bytes, data format
__device__ static inline rsrc_words_t make_rsrc_words(const void* p, uint32_t bytes) {
  const uint64_t b = reinterpret_cast<uint64_t>(p);
  rsrc_words_t w;
  w.x = (int)(uint32_t)b;
  w.y = (int)((uint32_t)(b >> 32) & 0xffffu);
  w.z = (int)bytes;
  w.w = 0x00020000;
  return w;
}
__device__ static inline void load_lds16(rsrc_words_t w, uint32_t lds_addr, uint32_t byte_off) {
  asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"(lds_addr), "v"(byte_off), "s"(w)
               : "memory");  // M0 cannot be named as a clobber: the compiler treats it as a reserved register (it rejects
                             // "m0" in a clobber list as such), i.e. it never keeps a value in M0 from one statement to
                             // the next and writes M0 itself right before each of its own uses
}
// wait until at most N of this wave's vector memory loads are outstanding
template <int N>
__device__ static inline void wait_vmem() {
  static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
  asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory");
}

// the same, and until this wave's LDS reads are done; then the workgroup's barrier.  (Builtins, so that the compiler's own
// count of outstanding LDS reads starts from zero behind it; the empty statements keep memory accesses on their side.)
template <int N>
__device__ static inline void wait_step() {
  static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
  asm volatile("" : : : "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));   // vmcnt(N) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" : : : "memory");
}

}  // namespace cd
