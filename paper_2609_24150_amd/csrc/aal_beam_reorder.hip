// The states of beams after a selection (aal_beam_reorder):
//
//   dst[b, j] = src[b, parents[b, j]]
//
// for a list of arrays, in one launch for up to 40 of them.  A thread has one piece (16 bytes, fewer at a segment's
// end) at one place of a request's slots: it loads that place of every slot's
// parent, then stores them, so that in place no slot is overwritten before it has been
// read, and nothing waits for another thread.  In place, slots that are their own parent are
// neither loaded nor stored.  Bound by memory: a write for each byte that moves, and a read for each that is some slot's parent.  0.8 GB of slots in
// place 275 us, of which 0.55 GB are read, 4.9 TB/s; into other buffers 1.2 GB of slots 424 us (318 and 450 with stores that stay in the caches); segments of 1,000 bytes
// from anywhere 4.6 TB/s (2.6 in pieces of 4 bytes).
#include "aal_beam.h"
#include "aal_device.h"

namespace aal {
namespace {

// States of a launch: their descriptions are kernel arguments, under 4 KiB, and under 1 KiB where there are few, which is
// less to hand over.
constexpr int kStates = 40, kFew = 8;

// Where so many pieces are to be looked at in place, threads have several of few slots each, since workgroups that find
// nothing to move cost as long as they take to start: 11 requests of 2 beams that all stay, 1.8 GB, 53 us with 8 pieces a
// thread, 405 with one; half of them moved 347 and 595; 8 requests of 4, half of 1.6 GB moved, 273 with 4 and 330 with one.
// Of many slots a thread has enough (8 slots: 570 us with 8 pieces, 520 with 2, 509 with one), and so has it into other buffers
// (325 and 277).
constexpr int64_t kManyPieces = int64_t(1) << 22;

template <int STATES>
struct ReorderParams {
  BeamState s[STATES];
  int64_t end[STATES];      // workgroups up to and with each state's
  uint32_t chunks[STATES];  // workgroups per request
  int64_t first;             // workgroup that the launch starts with
  int n_states, W, n;
  int rounds;                // pieces of a thread, one after the other
  const int32_t* parents;
};

typedef u32x4 u32x4_e1 __attribute__((aligned(1)));
typedef u32x2 u32x2_e1 __attribute__((aligned(1)));
typedef uint32_t u32_e1 __attribute__((aligned(1)));
typedef uint16_t u16_e1 __attribute__((aligned(1)));

// At any address: accesses of up to 16 bytes take those.
__device__ __forceinline__ void load_at(u32x4& r, const uint8_t* at) { r = *reinterpret_cast<const u32x4_e1*>(at); }
__device__ __forceinline__ void load_at(u32x2& r, const uint8_t* at) { r = *reinterpret_cast<const u32x2_e1*>(at); }
__device__ __forceinline__ void load_at(uint32_t& r, const uint8_t* at) { r = *reinterpret_cast<const u32_e1*>(at); }
__device__ __forceinline__ void load_at(uint16_t& r, const uint8_t* at) { r = *reinterpret_cast<const u16_e1*>(at); }
__device__ __forceinline__ void load_at(uint8_t& r, const uint8_t* at) { r = *at; }
__device__ __forceinline__ void store_at(u32x4 r, uint8_t* at) { __builtin_nontemporal_store(r, reinterpret_cast<u32x4_e1*>(at)); }
__device__ __forceinline__ void store_at(u32x2 r, uint8_t* at) { __builtin_nontemporal_store(r, reinterpret_cast<u32x2_e1*>(at)); }
__device__ __forceinline__ void store_at(uint32_t r, uint8_t* at) { __builtin_nontemporal_store(r, reinterpret_cast<u32_e1*>(at)); }
__device__ __forceinline__ void store_at(uint16_t r, uint8_t* at) { __builtin_nontemporal_store(r, reinterpret_cast<u16_e1*>(at)); }
__device__ __forceinline__ void store_at(uint8_t r, uint8_t* at) { __builtin_nontemporal_store(r, at); }

// VB: bytes of a piece.  WHOLE: segments are a number of them.  NB: slots held at a time (in place: all of them)
template <int VB, bool WHOLE, int NB, bool IN_PLACE, int STATES>
__global__ __launch_bounds__(256) void k_beam_reorder(ReorderParams<STATES> p) {
  const int64_t block = p.first + blockIdx.x;
  int k = 0;
  while (k + 1 < p.n_states && block >= p.end[k]) ++k;
  const BeamState& s = p.s[k];
  const int64_t at = block - (k ? p.end[k - 1] : 0);
  const int64_t b = at / p.chunks[k];
  const int32_t* parents = p.parents + b * p.n;
  if constexpr (IN_PLACE) {
    bool any = false;
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (j < p.n) any |= parents[j] >= 0 && parents[j] < p.W && parents[j] != j;
    if (!any) return;
  }
  const int64_t per = (s.segment_bytes + VB - 1) / VB, i0 = (at % p.chunks[k]) * 256 * p.rounds + threadIdx.x;
  for (int round = 0; round < p.rounds; ++round) {
    const int64_t i = i0 + round * 256;
    if (i >= per * s.segments) return;
    const int64_t seg = i / per, off = (i - seg * per) * VB;
    const uint8_t* src = s.src + b * s.src_request + seg * s.src_segment + off;
    uint8_t* dst = s.dst + b * s.dst_request + seg * s.dst_segment + off;
    // the bytes of a T in every slot
    auto move = [&](auto like) {
      using T = decltype(like);
      for (int j0 = 0; j0 < p.n; j0 += NB) {
        T r[NB];
        int from[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          from[j] = -1;
          if (j0 + j < p.n) {
            from[j] = parents[j0 + j];
            if (from[j] >= p.W || (IN_PLACE && from[j] == j0 + j)) from[j] = -1;
          }
          if (from[j] >= 0) load_at(r[j], src + from[j] * s.src_beam);
        }
#pragma unroll
        for (int j = 0; j < NB; ++j)
          if (from[j] >= 0) store_at(r[j], dst + (j0 + j) * s.dst_beam);
      }
      src += sizeof(T);
      dst += sizeof(T);
    };
    const int64_t left = s.segment_bytes - off;
    if (WHOLE || left >= VB) {
      if constexpr (VB == 16)
        move(u32x4{});
      else
        move(u32x2{});
      continue;
    }
    // a segment's end, which no other thread has any of
    if (VB == 16 && (left & 8)) move(u32x2{});
    if (left & 4) move(uint32_t{});
    if (left & 2) move(uint16_t{});
    if (left & 1) move(uint8_t{});
  }
}

template <int VB, bool WHOLE, int NB, int STATES>
void enqueue(const ReorderParams<STATES>& p, unsigned grid, bool in_place, hipStream_t stream) {
  if (in_place)
    k_beam_reorder<VB, WHOLE, NB, true><<<grid, 256, 0, stream>>>(p);
  else if constexpr (NB <= 32)
    k_beam_reorder<VB, WHOLE, NB, false><<<grid, 256, 0, stream>>>(p);
}

template <bool WHOLE, int STATES>
void enqueue_slots(const ReorderParams<STATES>& p, unsigned grid, bool in_place, hipStream_t stream) {
  if (p.n <= 4)
    enqueue<16, WHOLE, 4>(p, grid, in_place, stream);
  else if (p.n <= 8)
    enqueue<16, WHOLE, 8>(p, grid, in_place, stream);
  else if (p.n <= 16)
    enqueue<16, WHOLE, 16>(p, grid, in_place, stream);
  else if (p.n <= 32 || !in_place)
    enqueue<16, WHOLE, 32>(p, grid, in_place, stream);
  else
    enqueue<8, WHOLE, 64>(p, grid, in_place, stream);
}

// The next states whose segments are a number of 16 bytes, or are not, from number `next` on, as many as a launch takes.
template <int STATES>
void launch_some(const ReorderArgs& a, bool whole, int rounds, int& next) {
  // slots beyond 32 in place are held in pieces of 8 bytes: 128 registers
  const int bytes = a.in_place && a.n > 32 ? 8 : 16;
  ReorderParams<STATES> p;
  p.n_states = 0;
  p.first = 0;
  p.W = a.W;
  p.n = a.n;
  p.parents = a.parents;
  p.rounds = rounds;
  int64_t total = 0;
  for (; next < a.n_states && p.n_states < STATES; ++next) {
    const BeamState& s = a.states[next];
    if (s.segments == 0 || s.segment_bytes == 0 || (s.segment_bytes % 16 == 0) != whole) continue;
    const int64_t chunks = (s.segments * ((s.segment_bytes + bytes - 1) / bytes) + 256 * rounds - 1) / (256 * rounds);
    total += a.B * chunks;
    p.s[p.n_states] = s;
    p.chunks[p.n_states] = uint32_t(chunks);
    p.end[p.n_states++] = total;
  }
  // a launch holds fewer than 2^32 threads
  for (; p.first < total; p.first += int64_t(1) << 23) {
    const unsigned grid = unsigned(total - p.first < (int64_t(1) << 23) ? total - p.first : int64_t(1) << 23);
    if (whole)
      enqueue_slots<true>(p, grid, a.in_place, a.stream);
    else
      enqueue_slots<false>(p, grid, a.in_place, a.stream);
  }
}

}  // namespace

hipError_t launch_beam_reorder(const ReorderArgs& a) {
  if (a.in_place && a.W == 1) return hipSuccess;  // its own parent, or none
  int64_t pieces = 0;
  for (int i = 0; i < a.n_states; ++i) pieces += a.B * a.states[i].segments * ((a.states[i].segment_bytes + 15) / 16);
  const int rounds = !a.in_place || pieces <= kManyPieces ? 1 : a.n <= 2 ? 8 : a.n <= 4 ? 4 : a.n <= 8 ? 2 : 1;
  for (bool whole : {true, false})
    for (int next = 0; next < a.n_states;)
      if (a.n_states - next <= kFew)
        launch_some<kFew>(a, whole, rounds, next);
      else
        launch_some<kStates>(a, whole, rounds, next);
  return hipGetLastError();
}

}  // namespace aal
