// The states of beams after a selection (aal_beam_reorder):
//
//   dst[b, j] = src[b, parents[b, j]]
//
// for a list of arrays, in one launch for up to 40 of them.  A thread has one piece (16 bytes, or what
// addresses and strides divide) at one place of a request's slots: it loads that place of every slot's
// parent, then stores them, so that in place no slot is overwritten before it has been
// read, and nothing waits for another thread.  In place, slots that are their own parent are
// neither loaded nor stored.  Bound by memory: two bytes of traffic for each byte that moves.  0.8 GB of caches in place 300
// us, 5.4 TB/s, into other buffers 424 us for 1.2 GB (318 and 450 with stores that stay in the caches).
#include "aal_beam.h"
#include "aal_device.h"

namespace aal {
namespace {

// States of a launch: their descriptions are kernel arguments, under 4 KiB, and under 1 KiB where there are few, which is
// less to hand over.
constexpr int kStates = 40, kFew = 8;

template <int STATES>
struct ReorderParams {
  BeamState s[STATES];
  int64_t end[STATES];      // workgroups up to and with each state's
  uint32_t chunks[STATES];  // workgroups per request
  int64_t first;             // workgroup that the launch starts with
  int n_states, W, n;
  const int32_t* parents;
};

template <int VB> struct PieceOf;
template <> struct PieceOf<16> { using type = u32x4; };
template <> struct PieceOf<8> { using type = u32x2; };
template <> struct PieceOf<4> { using type = uint32_t; };
template <> struct PieceOf<1> { using type = uint8_t; };

// VB: bytes of a piece, NB: slots held at a time (in place: all of them)
template <int VB, int NB, bool IN_PLACE, int STATES>
__global__ __launch_bounds__(256) void k_beam_reorder(ReorderParams<STATES> p) {
  using T = typename PieceOf<VB>::type;
  const int64_t block = p.first + blockIdx.x;
  int k = 0;
  while (k + 1 < p.n_states && block >= p.end[k]) ++k;
  const BeamState& s = p.s[k];
  const int64_t at = block - (k ? p.end[k - 1] : 0);
  const int64_t b = at / p.chunks[k];
  const int64_t per = s.segment_bytes / VB, i = (at % p.chunks[k]) * 256 + threadIdx.x;
  if (i >= per * s.segments) return;
  const int64_t seg = i / per, off = (i - seg * per) * VB;
  const uint8_t* src = s.src + b * s.src_request + seg * s.src_segment + off;
  uint8_t* dst = s.dst + b * s.dst_request + seg * s.dst_segment + off;
  const int32_t* parents = p.parents + b * p.n;
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
      if (from[j] >= 0) r[j] = *reinterpret_cast<const T*>(src + from[j] * s.src_beam);
    }
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (from[j] >= 0) __builtin_nontemporal_store(r[j], reinterpret_cast<T*>(dst + (j0 + j) * s.dst_beam));
  }
}

template <int VB, int NB, int STATES>
void enqueue(const ReorderParams<STATES>& p, unsigned grid, bool in_place, hipStream_t stream) {
  if (in_place)
    k_beam_reorder<VB, NB, true><<<grid, 256, 0, stream>>>(p);
  else if constexpr (NB <= 32)
    k_beam_reorder<VB, NB, false><<<grid, 256, 0, stream>>>(p);
}

// The piece that all of a state's addresses, strides and sizes are multiples of.
int piece_of(const BeamState& s, int W, int n, int64_t B) {
  uint64_t bits = uint64_t(s.segment_bytes) | uint64_t(reinterpret_cast<uintptr_t>(s.src)) |
                  uint64_t(reinterpret_cast<uintptr_t>(s.dst));
  if (W > 1 || n > 1) bits |= uint64_t(s.src_beam) | uint64_t(s.dst_beam);
  if (B > 1) bits |= uint64_t(s.src_request) | uint64_t(s.dst_request);
  if (s.segments > 1) bits |= uint64_t(s.src_segment) | uint64_t(s.dst_segment);
  return bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 1;
}

template <int VB, int STATES>
void enqueue_piece(const ReorderParams<STATES>& p, unsigned grid, bool in_place, hipStream_t stream) {
  if (p.n <= 4)
    enqueue<VB, 4>(p, grid, in_place, stream);
  else if (p.n <= 8)
    enqueue<VB, 8>(p, grid, in_place, stream);
  else if (p.n <= 16)
    enqueue<VB, 16>(p, grid, in_place, stream);
  else if (p.n <= 32 || !in_place)
    enqueue<VB, 32>(p, grid, in_place, stream);
  else
    enqueue<VB, 64>(p, grid, in_place, stream);
}

// The next states of that piece, from number `next` on, as many as a launch takes.
template <int STATES>
void launch_some(const ReorderArgs& a, int piece, int& next) {
  // slots beyond 32 in place are held in pieces of 8 bytes: 128 registers
  const int bytes = piece == 16 && a.in_place && a.n > 32 ? 8 : piece;
  ReorderParams<STATES> p;
  p.n_states = 0;
  p.first = 0;
  p.W = a.W;
  p.n = a.n;
  p.parents = a.parents;
  int64_t total = 0;
  for (; next < a.n_states && p.n_states < STATES; ++next) {
    const BeamState& s = a.states[next];
    if (s.segments == 0 || s.segment_bytes == 0 || piece_of(s, a.W, a.n, a.B) != piece) continue;
    const int64_t chunks = (s.segments * (s.segment_bytes / bytes) + 255) / 256;
    total += a.B * chunks;
    p.s[p.n_states] = s;
    p.chunks[p.n_states] = uint32_t(chunks);
    p.end[p.n_states++] = total;
  }
  // a launch holds fewer than 2^32 threads
  for (; p.first < total; p.first += int64_t(1) << 23) {
    const unsigned grid = unsigned(total - p.first < (int64_t(1) << 23) ? total - p.first : int64_t(1) << 23);
    if (bytes == 16)
      enqueue_piece<16>(p, grid, a.in_place, a.stream);
    else if (bytes == 8)
      enqueue<8, 64>(p, grid, true, a.stream);
    else if (bytes == 4)
      enqueue_piece<4>(p, grid, a.in_place, a.stream);
    else
      enqueue_piece<1>(p, grid, a.in_place, a.stream);
  }
}

}  // namespace

hipError_t launch_beam_reorder(const ReorderArgs& a) {
  for (int piece : {16, 4, 1})
    for (int next = 0; next < a.n_states;)
      if (a.n_states - next <= kFew)
        launch_some<kFew>(a, piece, next);
      else
        launch_some<kStates>(a, piece, next);
  return hipGetLastError();
}

}  // namespace aal
