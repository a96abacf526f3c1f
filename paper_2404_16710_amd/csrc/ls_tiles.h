// Operand tiles that are sent straight into LDS, for the products of the prompt pass and of the head's training.
#ifndef LS_TILES_H_
#define LS_TILES_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

typedef unsigned int mm_u32x4 __attribute__((ext_vector_type(4)));

constexpr int MM_ROWB = 64;       // bytes of K per step and row

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// 64 lanes x 16 bytes from rsrc[voff + soff] to LDS at lds_addr + 16 * lane.
__device__ __forceinline__ void mm_request(uint32_t lds_addr, uint32_t voff, mm_u32x4 rsrc, uint32_t soff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :: "s"(lds_addr), "v"(voff), "s"(rsrc), "s"(soff) : "m0");   // (m0 is nobody's between two instructions)
}
#pragma clang diagnostic pop
// All but the N youngest requests of this wave have landed, its LDS reads are done, and so have everybody's.
template <int N>
__device__ __forceinline__ void mm_wait_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
}
__device__ __forceinline__ mm_u32x4 mm_rsrc(const void* base, uint32_t bytes) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  mm_u32x4 r;
  r[0] = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p);
  r[1] = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32) & 0xFFFF);
  r[2] = (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes);
  r[3] = 0x00020000u;
  // A buffer load may read a scalar register five wait states after a vector instruction (readfirstlane) wrote it, and
  // the compiler does not count them in front of hand-written instructions.  (Today it makes these words with scalar
  // instructions, which need no wait.)
  asm volatile("s_nop 4" : "+s"(r));
  return r;
}

// Tile and split of a workgroup: dealt out die by die in panels of 4 tile columns like pf_tile_of, the splits of
// the whole product one after the other (workgroups that run together share K ranges as well as rows).
__device__ __forceinline__ void mm_tile_of(int MT, int NT, int splits, int& tm, int& tn, int& split) {
  constexpr int NX = 8, PN = 4;
  const int tiles = MT * NT, total = tiles * splits, id = (int)blockIdx.x;
  const int x = id % NX;
  const int q = total / NX, rem = total % NX;
  const int lin = x * q + (x < rem ? x : rem) + id / NX;
  split = lin / tiles;
  const int l = lin - split * tiles;
  const int panel = l / (MT * PN), n_first = panel * PN;
  const int pw = NT - n_first < PN ? NT - n_first : PN;
  const int rr = l - panel * MT * PN;
  tm = rr / pw;
  tn = n_first + (rr - tm * pw);
}

// Pairs of steps in the ring.  The 128 x 128 and the 64 x 64 tile leave room for a second workgroup on the compute unit
// (64 KB of ring each); the others have the LDS of theirs to themselves (128 KB with a 256 x 256 tile, 144 with 256 x 128,
// 96 with 128 x 64 and 64 x 128, which have four pairs in flight instead of a neighbour).
template <int RM, int RN> constexpr int mm_pairs() { return RM + RN >= 16 ? 2 : RM + RN >= 12 ? 3 : RM + RN >= 8 ? 2 : 4; }
template <int RM, int RN> constexpr int mm_smem_bytes() { return (RM + RN) * 32 * MM_ROWB * 2 * mm_pairs<RM, RN>(); }

extern __shared__ __align__(1024) char mm_smem[];

#endif
