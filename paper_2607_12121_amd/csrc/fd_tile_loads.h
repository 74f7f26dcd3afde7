// What the tiled products of 8-bit rows share: rows in pieces of 32 bytes, loads from memory into LDS and the waits
// that count them.
#pragma once

#include "fd_common.h"

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));

// 32 bytes at p + k of a row of K bytes, K a multiple of 16; past its end the last 16 bytes again, for inside() to clear.
struct Piece { uint4 lo, hi; };
FD_DEVICE Piece load32(const uint8_t* p, int k, int K) {
  return {*reinterpret_cast<const uint4*>(p + min(k, K - 16)), *reinterpret_cast<const uint4*>(p + min(k + 16, K - 16))};
}
FD_DEVICE i32x8_t inside(const Piece& x, int k, int K) {
  const uint4 none = make_uint4(0, 0, 0, 0), lo = k < K ? x.lo : none, hi = k + 16 < K ? x.hi : none;
  return i32x8_t{static_cast<int>(lo.x), static_cast<int>(lo.y), static_cast<int>(lo.z), static_cast<int>(lo.w),
                 static_cast<int>(hi.x), static_cast<int>(hi.y), static_cast<int>(hi.z), static_cast<int>(hi.w)};
}

typedef __attribute__((address_space(3))) void* lds_ptr_t;

FD_DEVICE i32x4_t buffer_of(const void* base, uint32_t bytes = 0x7fffffffu) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  return i32x4_t{static_cast<int>(static_cast<uint32_t>(p)), static_cast<int>(static_cast<uint32_t>(p >> 32) & 0xffffu), static_cast<int>(bytes), 0x00020000};
}
constexpr uint32_t kNowhere = 0x80000000u;   // an offset past every buffer: loads read zeros, stores are dropped
// Cache policy of wide results: non-temporal, so that they leave the L2 to the operands (9828 x 4608 x 1536 to bf16
// 77.4 -> 74.8 us, x 1536 x 6144 84.3 -> 79.7; codes, a quarter to a half of the bytes, the same either way).
constexpr int kStream = 2;
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
// A store of four fp32 per lane at voff + soff, the sum in a vector register and none in the scalar one.  A store of more
// than 8 bytes reads its data over several clocks, and a vector instruction right behind it that writes these registers has to
// wait two states; the compiler puts them there only where the store has no scalar offset.  With one, the first of the
// four values came out as the next row's raw sum (9728 of 16.8 million, 8192 x 2048 x 16).
template <class Rsrc>
FD_DEVICE void store_f4(float a, float b, float c, float d, Rsrc y, uint32_t voff, uint32_t soff) {
  __builtin_amdgcn_raw_buffer_store_b128(u32x4_t{__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d)}, y,
                                         static_cast<int>(voff + soff), 0, kStream);
}
// 16 (4) bytes per lane from buffer offset voff + soff into LDS at lds + MORE + 16 (4) * lane.  In assembly so that
// the compiler does not wait for it before unrelated LDS reads.  A load to LDS takes M0 one wait state after its write.
template <int MORE>
FD_DEVICE void dma16(uint32_t lds, uint32_t voff, i32x4_t rsrc, uint32_t soff) {
  asm volatile("s_add_u32 m0, %0, %4\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "s"(lds), "v"(voff), "s"(rsrc), "s"(soff), "n"(MORE) : "scc");
}
FD_DEVICE void dma4(uint32_t lds, uint32_t voff, i32x4_t rsrc, uint32_t soff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" : : "s"(lds), "v"(voff), "s"(rsrc), "s"(soff));
}
// This wave's LDS reads are done; then the barrier.
FD_DEVICE void wait_reads_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }
// ... and at most N of its vector memory operations are in flight (N + MORE where `more`).  One block of assembly:
// a branch around the wait would end the basic block, across which the compiler moves the products.
template <int N, int MORE>
FD_DEVICE void wait_barrier(int more) {
  static_assert(N + MORE < 64, "the counter's range");
  asm volatile(
      "s_waitcnt vmcnt(%1) lgkmcnt(0)\n\t"
      "s_cmp_lg_u32 %0, 0\n\t"
      "s_cbranch_scc1 .Lfd_wait_%=\n\t"
      "s_waitcnt vmcnt(%2)\n"
      ".Lfd_wait_%=:\n\t"
      "s_barrier"
      :
      : "s"(more), "n"(N + MORE), "n"(N)
      : "memory", "scc");
}

}  // namespace
