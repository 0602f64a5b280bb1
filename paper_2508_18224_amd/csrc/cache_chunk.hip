// Attention of pieces of prompts over a paged cache (nsa_sel_cache_attention_chunk): every key, or a window, for many new tokens of a sequence at a time.
//
// S = Q K^T, P = softmax(S), O = P V in one pass over the keys with the running maximum and sum of a row.  A key of a KV head is used by g rows of every token that sees
// it, so a workgroup takes 256 rows (256 / g consecutive tokens of a sequence) of a KV head, a unit, and walks the keys in pieces of 64: eight wavefronts of 32 rows, two to a
// SIMD, each with its Q and its output in registers, share a piece's K and V in LDS.  A piece is 32 KB and 8.4 MFLOP, 2048 clocks of the matrix pipes; reading its operands takes the
// LDS as long.
//
// What bounds it is the vector phase, and power: a wavefront's vector phase takes 1810 clocks, its matrix phase, beside another's vector phase, 1610, both together 3880, at 2.0 to 2.1 GHz
// with random numbers.  (The products of a piece and their operand reads alone: 1.23 us, at 1.7 GHz; the whole: 1.82.)  2048 new tokens of 32 heads behind 32768 keys (8 KV heads) take 0.99 to
// 1.02 ms by card, 1.11 to 1.14 PFLOP/s; a large library product reaches 1.6.
//
// A page of 16 tokens or more is a run of memory, so the eight rows that a wavefront moves of a piece's K and V are always one page's: which one is looked up for 64 pieces
// at a time, a piece a lane, and in the loop, which asks three pieces ahead, again after 61.
//
// Probabilities are rounded to bf16 for their product, as in the prompt's own attention (their relative error counts, and is the same for all of them); the sums they are
// divided by are not.
#include <type_traits>

#include "cache_checks.h"
#include "dense_piece.h"

namespace nsa {
namespace {

constexpr int kChunkWaves = 8, kChunkRows = 32 * kChunkWaves, kChunkThreads = 64 * kChunkWaves;
constexpr int kStages = 4;  // tiles of K, and of V: one more than a piece that is asked for two before it is used needs, so that nobody waits for the tile to be free
constexpr int kChunkV = kStages * kPieceBytes, kChunkLds = 2 * kStages * kPieceBytes + 64;
constexpr int kSlots = 256;  // workgroups that share all units' pieces evenly, at most
// What a unit costs beside its pieces, in pieces: its Q, its pages, the first and the last piece, its result, 10 to 12 us for 1.8 of a piece.  (A whole prompt of 8192 tokens: 1300 us
// with none of it counted, 1023 with 5, 1004 with 6, 1013 with 8, when a piece took 1.7.)
constexpr int kUnitCost = 6;
constexpr int kLeastSpan = 2, kLeastShare = 6;  // (16 tokens behind 4080 keys: 23.6 us with 5 or 6 to a workgroup, 24.7 with 7, 28.5 with 12)
constexpr int kChunkJoinThreads = 512;
static_assert(kChunkRows * kPieceRow <= kChunkLds, "the result must fit where the tiles were");

struct ChunkArgs {
  const void* Q;
  int32_t window;
  float scale;
  const float* gate;
  const void* o_acc;
  void* O;
  float* LSE;
  int32_t tok;       // tokens of a unit
  uint32_t g_magic;  // see div_g
  int32_t units;     // of a KV head, at most
  int32_t slots;     // workgroups, a multiple of 8
  // parts of units: part 2 w of workgroup w for the unit that others begin, 2 w + 1 for the one that it begins and others finish
  float* part;       // [2 slots][8 wavefronts][16][64 lanes][4]: the sums as the lanes hold them
  float2* part_ml;   // [2 slots][256] (reference, sum)
  struct Joint* joints;  // [slots]
};

// A kernel's arguments, read anew from where the launch put them wherever this is called: held in registers through the loop over the keys, they would crowd out what that needs.
struct Args {
  Cache C;
  ChunkArgs A;
};
__device__ __forceinline__ const Args& arguments() {
  auto p = (const __attribute__((address_space(4))) Args*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const Args*)p;
}

// Of every workgroup: the unit that it has the first pieces of and not the last ones, if there is one (else parts is 0).  Its parts are in slot `first`, in the first slots of the next
// workgroups.
struct Joint {
  int t0, nt, j, parts, first, second, pad[2];
};

// A unit of the call: nt consecutive new tokens t0.. of sequence s, the first of them at `place`, and KV head j; s < 0 where there is none.
struct Unit {
  int s, t0, nt, place, j;
};
__device__ __forceinline__ int64_t first_unit(const Cache& C, const ChunkArgs& A, int s) {
  // a sequence's units start at floor(cu / tok) + s: room for all of them without a scan over the batch
  return (int64_t)(C.cu ? C.cu[s] / A.tok : 0) + s;
}
__device__ __forceinline__ Unit unit_of(const Cache& C, const ChunkArgs& A, int s, int i, int j) {
  Unit W;
  const int c0 = C.cu ? C.cu[s] : s, n = C.cu ? C.cu[s + 1] - c0 : 1, i0 = i * A.tok;
  W.s = s;
  W.j = j;
  W.t0 = c0 + i0;
  W.nt = min(min(A.tok, n - i0), C.T - W.t0);
  W.place = max(C.kv_len[s], kLeastLength) - n + i0;
  if (W.nt <= 0 || W.t0 < 0) W.s = -1;
  return W;
}
// The pieces that anything of the unit sees: [first, first + count).
__device__ __forceinline__ int2 pieces_of(const Cache& C, const ChunkArgs& A, const Unit& W) {
  const int hi = min(W.place + W.nt, C.max_pages << C.page_log2), lo = A.window > 0 ? window_start(W.place, A.window) : 0;
  const int first = lo / 64;
  return {first, max((hi + 63) / 64 - first, 0)};
}

// Rows of 128 bf16 lie in LDS unpadded, the 16-byte chunk c of row r at place c ^ piece_turn(r).  Then the 64 banks are all in use with every read of a piece: keys' reads, where the hardware
// serves lanes 0-3, 12-15 and 20-27 at once (rows 0-3 and 12-15 of a chunk, rows 4-11 of the next one: both sets of turns are closed under a flip of the lowest bit), values' reads, where it
// serves two chunks of eight rows (the turns of rows 0-7, and of rows 8-15, differ above the lowest bit), and writes of sixteen 8-bit values a lane (see put).  (Rows turned as the other
// kernels have them: every second cycle of the LDS a conflict.)
__device__ __forceinline__ int piece_turn(int r) { return ((r & 8 ? ~r : r) & 7) << 1 | (r >> 3 & 1); }
// Operand reads of a piece: they differ in bits that are flipped, and take no registers when made anew from one address.
// Keys: of 16 rows, lane l the row l % 16, channels 8 (l / 16) .. of step s of the contraction.  Values: transposed, 16 channels, keys 4 (l / 16) .. of two groups of 16.
__device__ __forceinline__ bf16x8 key_operand(uint32_t at, int s, int group) { return lds_read_frag((at ^ (s << 6)) + 16 * group * kPieceRow); }
__device__ __forceinline__ bf16x8 value_operand(uint32_t at, int sp, int db) {
  const uint32_t a = (at ^ (db << 5)) + 32 * sp * kPieceRow;
  const bf16x4 a0 = lds_read_tr_at(a), a1 = lds_read_tr_at(a + 16 * kPieceRow);
  return __builtin_shufflevector(a0, a1, 0, 1, 2, 3, 4, 5, 6, 7);
}

// threadIdx.x & 63, made anew wherever it is asked for: what derives from it need not be kept.
__device__ __forceinline__ int own_lane() {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  return tid & 63;
}
// This lane's row x of a wavefront's 32, a lane having two, l % 16 and 16 on: token of the unit and row of Q and O.  Lanes past the last row go along with it.
struct LaneRow {
  int r, token;
  int64_t row;
  bool here;
};
__device__ __forceinline__ LaneRow lane_row(const Cache& C, const ChunkArgs& A, const Unit& W, int wave, int x) {
  LaneRow L;
  const int rows = W.nt * C.g;
  L.r = 32 * wave + 16 * x + (own_lane() & 15);
  L.here = L.r < rows;
  const int rc = min(L.r, rows - 1);
  L.token = div_g(rc, C.g, A.g_magic);
  L.row = (int64_t)(W.t0 + L.token) * C.hq + W.j * C.g + (rc - L.token * C.g);
  return L;
}

// What a row's exponents are taken against: its running maximum times scale * log2(e), rounded, and `ref` is that rounded number, so that alpha, what the sums so far are to be
// multiplied by, is exactly 1 while the maximum stays.  With the maximum itself kept, and rounded anew for every piece, alpha would be 1 but for that rounding's error, the same
// for every piece: over 2048 pieces up to 1.7e-4 of the sum.  It takes in every new
// maximum, so that the largest probability so far is 1, which bf16 holds exactly.  (With a reference that may lag by 2^6 the sums are rescaled in 1 instead of 23 % of the pieces: 2048 tokens behind
// 32768 keys 948 us against 995, a whole prompt of 8192 970 against 1051, ragged pieces in 8 bits 469 against 508; but O's error is 5 to 7 % larger with scores of unit spread, 14 to 22 % with twice that.)
__device__ __forceinline__ float finite_reference(float ref) { return ref == -INFINITY ? 0.f : ref; }
__device__ __forceinline__ float new_reference(float m, float& ref, float& alpha) {
  const float now = fmaxf(m, ref), mc = finite_reference(now);
  alpha = __builtin_amdgcn_exp2f(ref - mc);  // exp2(-inf) = 0 on the first piece with a score
  ref = now;
  return mc;
}

// The two rows of a lane are those of three others too (l % 16).  What there is one of for a row, the lower half of the lanes has for the first rows, the upper half for the second ones.
struct Two {
  float x, y;
};
__device__ __forceinline__ Two swap_32(float a, float b) {  // lower half: (a, a of the lane 32 on); upper half: (b of the lane 32 back, b)
  const auto z = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false, false);
  const uint32_t low = z[0], high = z[1];  // (by way of integers: a bit cast of an element takes the first one)
  return {__builtin_bit_cast(float, low), __builtin_bit_cast(float, high)};
}
__device__ __forceinline__ Two both_rows(float x) { return swap_32(x, x); }  // the first rows' and the second rows', in all lanes
__device__ __forceinline__ Two swap_16(float a) {
  const uint32_t x = __builtin_bit_cast(uint32_t, a);
  const auto z = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  const uint32_t low = z[0], high = z[1];
  return {__builtin_bit_cast(float, low), __builtin_bit_cast(float, high)};
}
__device__ __forceinline__ float row_max(float a, float b) {
  const Two h = swap_32(a, b), q = swap_16(fmaxf(h.x, h.y));
  return fmaxf(q.x, q.y);
}
__device__ __forceinline__ float row_sum(float a, float b) {
  const Two h = swap_32(a, b), q = swap_16(h.x + h.y);
  return q.x + q.y;
}

// Eight rows of a wavefront straight to LDS (see load_to_lds), four a load, the second four 1 KB on on both sides: the instruction's offset counts for both.
__device__ __forceinline__ void load_rows_to_lds(u32x4 b, uint32_t lds, uint32_t off, uint32_t off2) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %3, 0 offen lds\n\tbuffer_load_dwordx4 %2, %3, 0 offen offset:1024 lds"
               :: "s"(lds), "v"(off), "v"(off2), "s"(b) : "memory", "m0");
}

// ---- the products of a matrix phase, in order: those of the scores S^T = K Q^T of a piece with 16 operands, those of O^T += V^T P^T of the one before with 16 more, two rows' groups for
// each.  16 x 16 x 32: with random numbers they and their reads take 1.23 us a piece alone where those of 32 x 32 x 16 take 1.36, for less power (and 1.34 where a wavefront has 64 rows and
// half the reads); in the whole kernel, where they take twice the issue slots, that is 1 %.  A wavefront issues in order: operand reads go kAhead operands ahead, two at a time.
constexpr int kAhead = 4;
__device__ __forceinline__ bf16x8 phase_operand(uint32_t k, uint32_t v, int i) {
  return i < 16 ? key_operand(k, i >> 2, i & 3) : value_operand(v, (i - 16) >> 3, (i - 16) & 7);
}
template <bool kScores>
__device__ __forceinline__ void first_operands(uint32_t k, uint32_t v, bf16x8 (&frag)[kAhead]) {
#pragma unroll
  for (int i = 0; i < kAhead; ++i) frag[i] = phase_operand(k, v, (kScores ? 0 : 16) + i);
}
// s[m][x][e]: the score of key 16 m + 4 (l / 16) + e with row x of this lane; oacc[db][x][e]: channel 16 db + 4 (l / 16) + e of it
template <bool kScores, bool kValues, class Beside>
__device__ __forceinline__ void matrix_phase(uint32_t k, uint32_t v, const bf16x8 (&qf)[2][4], const bf16x8 (&pf)[2][2], f32x4 (&s)[4][2], f32x4 (&oacc)[8][2],
                                             bf16x8 (&frag)[kAhead], Beside beside) {
  constexpr int kFirst = kScores ? 0 : 16, kLast = kValues ? 32 : 16;
  if constexpr (kScores) {
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int x = 0; x < 2; ++x) s[m][x] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
#pragma unroll
  for (int i0 = kFirst; i0 < kLast; i0 += 2) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = i0; i < i0 + 2; ++i)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if (i < 16) s[i & 3][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag[i % kAhead], qf[x][i >> 2], s[i & 3][x], 0, 0, 0);
        else oacc[i & 7][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(frag[i % kAhead], pf[x][(i - 16) >> 3], oacc[i & 7][x], 0, 0, 0);
      }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = i0; i < i0 + 2; ++i) {
      if (i + kAhead < kLast) frag[i % kAhead] = phase_operand(k, v, i + kAhead);
      beside(i);
    }
  }
  __builtin_amdgcn_sched_barrier(0);
}

// The part [begin, end) of a unit's pieces that a workgroup takes; if that is not all of them the sums go to slot `slot`.
struct Span {
  int begin, end, slot;
  bool whole;
};

template <bool kE4m3>
__device__ __forceinline__ void attend_unit(Unit W, Span P, char* smem) {
  const int lane = own_lane(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = lane >> 4;
  // the same in every lane, and said so: the buffers below are scalar
  W.s = __builtin_amdgcn_readfirstlane(W.s);
  W.t0 = __builtin_amdgcn_readfirstlane(W.t0);
  W.nt = __builtin_amdgcn_readfirstlane(W.nt);
  W.place = __builtin_amdgcn_readfirstlane(W.place);
  W.j = __builtin_amdgcn_readfirstlane(W.j);
  P.begin = __builtin_amdgcn_readfirstlane(P.begin);
  P.end = __builtin_amdgcn_readfirstlane(P.end);
  const int steps = P.end - P.begin;
  bool wave_on;                    // idle wavefronts still move K and V
  int first;                       // the first piece
  int least_hi, most_lo;           // what all rows of the wavefront see: rows are in the order of their tokens, the first one sees the fewest later keys
  float c2;
  const char *k_base, *v_base;
  f32x4 oacc[8][2];
  float ref, l_run[2];  // see new_reference, of the first or the second row; the rows' sums, of this lane's keys
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < 8; ++db)
#pragma unroll
      for (int x = 0; x < 2; ++x) oacc[db][x] = f32x4{0.f, 0.f, 0.f, 0.f};
    ref = -INFINITY;
    l_run[0] = l_run[1] = 0.f;
  };
  clear();
  bf16x8 qf[2][4];
  auto load_q = [&]() __attribute__((always_inline)) {
    const Cache& C = arguments().C;
    const ChunkArgs& A = arguments().A;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const bf16_t* src = (const bf16_t*)A.Q + lane_row(C, A, W, wave, x).row * kD + 8 * (own_lane() >> 4);
#pragma unroll
      for (int s = 0; s < 4; ++s) qf[x][s] = *reinterpret_cast<const bf16x8*>(src + 32 * s);
    }
  };
  load_q();
  {
    const Cache& C = arguments().C;
    const ChunkArgs& A = arguments().A;
    const int limit = C.max_pages << C.page_log2, rows = W.nt * C.g;
    first = pieces_of(C, A, W).x + P.begin;
    wave_on = 32 * wave < rows;
    least_hi = min(W.place + div_g(min(32 * wave, rows - 1), C.g, A.g_magic) + 1, limit);
    most_lo = A.window > 0 ? window_start(W.place + div_g(min(32 * wave + 31, rows - 1), C.g, A.g_magic), A.window) : 0;
    c2 = A.scale * 1.4426950408889634f;
    k_base = C.k;
    v_base = C.v;
  }
  const int v_row = ((lane & 15) >> 2) + 4 * part;
  const uint32_t k_at = lds_address(smem) + (lane & 15) * kPieceRow + ((part ^ piece_turn(lane & 15)) << 4);
  const uint32_t v_at = lds_address(smem + kChunkV) + v_row * kPieceRow + ((((lane & 3) >> 1) ^ piece_turn(v_row)) << 4) + 8 * (lane & 1);
  auto keys = [&](uint32_t off) __attribute__((always_inline)) { return k_at + off; };
  auto values = [&](uint32_t off) __attribute__((always_inline)) { return v_at + off; };

  // ---- pages: lane l knows those of piece base + l of the span, whose four 16-token groups may each have another one; this wavefront moves rows 8 wave.. of a piece
  constexpr int kRow = kE4m3 ? kD : kPieceRow;
  int base = 0;
  uint32_t off_lo, off_hi, word_of;  // byte offset of those rows of K and of V, and what is in a Move's word
  struct Move {
    uint32_t lo, hi;
    uint32_t word;  // bits 0-3: groups that have a page; 4: all rows of the wavefront see all of the piece; 8-11: rows to be moved; 16-23, 24-31: exponents of the page's scales
    __device__ __forceinline__ uint32_t bytes() const { return kE4m3 ? (word & 0xf00) >> 1 : word & 0xf00; }
    __device__ __forceinline__ float ks() const { return __builtin_bit_cast(float, (word >> 16 & 255) << 23); }
    __device__ __forceinline__ float vs() const { return __builtin_bit_cast(float, (word >> 24) << 23); }
    __device__ __forceinline__ const char* from(const char* base) const { return base + ((uint64_t)hi << 32 | lo); }
  };
  auto look_up = [&](int at) __attribute__((always_inline)) {
    const Cache& C = arguments().C;
    const int32_t* row = C.table + (int64_t)W.s * C.max_pages;
    base = at;
    const int step = at + lane, key = (first + step) * 64, mine = key + 8 * wave, limit = C.max_pages << C.page_log2;
    int page[5];  // as the table has them (one without columns has no pieces)
#pragma unroll
    for (int q = 0; q < 5; ++q) page[q] = row[min((q < 4 ? key + 16 * q : mine) >> C.page_log2, C.max_pages - 1)];
    asm volatile("" : "+v"(page[0]), "+v"(page[1]), "+v"(page[2]), "+v"(page[3]), "+v"(page[4]));  // all five at once
    auto there = [&](int k, int p) __attribute__((always_inline)) { return step < steps && k < limit && (uint32_t)p < (uint32_t)C.n_pages; };
    const int own = there(mine, page[4]) ? page[4] : -1;
    word_of = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) word_of |= there(key + 16 * q, page[q]) ? 1u << q : 0u;
    if (word_of == 15 && key + 64 <= least_hi && key >= most_lo) word_of |= 16;
    const int64_t head = (int64_t)max(own, 0) * C.hkv + W.j, off = ((head << C.page_log2) + (mine & ((1 << C.page_log2) - 1))) * kRow;
    off_lo = (uint32_t)off;
    off_hi = (uint32_t)(off >> 32);
    if (own >= 0) {
      word_of |= (uint32_t)min(max(min(W.place + W.nt, limit) - mine, 0), 8) << 8;
      if constexpr (kE4m3) {
        const uint32_t ks = __builtin_bit_cast(uint32_t, C.ks[head]), vs = __builtin_bit_cast(uint32_t, C.vs[head]);
        word_of |= (ks >> 23 & 255) << 16 | (vs >> 23 & 255) << 24;
      }
    }
    asm volatile("" : "+v"(off_lo), "+v"(off_hi), "+v"(word_of));  // no load of these is on its way where the tiles are waited for
  };
  auto word_at = [&](int step) __attribute__((always_inline)) { return (uint32_t)__builtin_amdgcn_readlane((int)word_of, step - base); };
  auto move_of = [&](int step) __attribute__((always_inline)) {
    return Move{(uint32_t)__builtin_amdgcn_readlane((int)off_lo, step - base), (uint32_t)__builtin_amdgcn_readlane((int)off_hi, step - base), word_at(step)};
  };
  // bf16: two loads of four rows, straight to LDS, lane l the place l % 16 of its row
  const uint32_t lds_rows = lds_address(smem) + 8 * wave * kPieceRow;
  const uint32_t move_off = (lane >> 4) * kPieceRow + (((lane & 15) ^ piece_turn(8 * wave + (lane >> 4))) << 4), move_off2 = move_off ^ 128;
  auto move = [&](const char* base, const Move& m, uint32_t lds_off) __attribute__((always_inline)) {
    const uint64_t at = (uint64_t)m.from(base);
    load_rows_to_lds(u32x4{(uint32_t)at, (uint32_t)(at >> 32), m.bytes(), 0x00020000u}, lds_rows + lds_off, move_off, move_off2);
  };
  // e4m3: eight rows into registers, to be written to LDS as bf16; eight lanes have a row, each eight channels of one half and then eight of the other, so that what they write at once
  // lies in different banks
  const int put_row = lane >> 3, half = put_row >> 1 & 1;
  const uint32_t fetch_off = put_row * kD + (lane & 7) * 8 + half * (kD / 2);
  auto fetch = [&](const char* base, const Move& m) __attribute__((always_inline)) {
    const auto rows = buffer_of(m.from(base), m.bytes());
    const auto x = __builtin_amdgcn_raw_buffer_load_b64(rows, fetch_off, 0, 0), y = __builtin_amdgcn_raw_buffer_load_b64(rows, fetch_off ^ (kD / 2), 0, 0);
    return u32x4{x[0], x[1], y[0], y[1]};
  };
  const uint32_t put_at = lds_rows + put_row * kPieceRow + (((8 * half + (lane & 7)) ^ piece_turn(8 * wave + put_row)) << 4);
  auto put = [&](u32x4 x, float scale, uint32_t lds_off) __attribute__((always_inline)) {
    const uint32_t at = put_at + lds_off;
    lds_write_16(at, eight_bf16(x[0], x[1], scale));
    lds_write_16(at ^ 128, eight_bf16(x[2], x[3], scale));
  };
  // a tile of K or V at once, in front of the main loop and in the simple one
  auto stage = [&](const char* base, const Move& m, float scale, uint32_t lds_off) __attribute__((always_inline)) {
    if constexpr (kE4m3) put(fetch(base, m), scale, lds_off);
    else move(base, m, lds_off);
  };

  // Scores -> what their exponents are taken against: keys that a row does not see become -inf, the row's maximum joins the running one.
  float alpha;
  Two mc;
  auto reference = [&](int step, uint32_t word, f32x4 (&s)[4][2]) __attribute__((always_inline)) {
    if (!(word & 16)) {
      const Cache& C = arguments().C;
      const int limit = C.max_pages << C.page_log2, window = arguments().A.window, key0 = (first + step) * 64 + 4 * (own_lane() >> 4);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int upto = W.place + lane_row(C, arguments().A, W, wave, x).token + 1;
        const int lim = min(upto, limit) - key0, lo = (window > 0 ? max(upto - window, 0) : 0) - key0;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
          const bool shown = word >> m & 1;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (16 * m + e >= (shown ? lim : INT32_MIN) || 16 * m + e < lo) s[m][x][e] = -INFINITY;
        }
      }
    }
    float most[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float m[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        m[h] = fmaxf(fmaxf(s[2 * h][x][0], s[2 * h][x][1]), s[2 * h][x][2]);
        m[h] = fmaxf(fmaxf(m[h], s[2 * h][x][3]), s[2 * h + 1][x][0]);
        m[h] = fmaxf(fmaxf(m[h], s[2 * h + 1][x][1]), s[2 * h + 1][x][2]);
      }
      most[x] = fmaxf(fmaxf(m[0], s[1][x][3]), fmaxf(m[1], s[3][x][3]));
    }
    mc = both_rows(new_reference(row_max(most[0], most[1]) * c2, ref, alpha));
  };
  // Scores -> probabilities as the operands of the two contraction steps of P V.
  auto probabilities = [&](const f32x4 (&s)[4][2], bf16x8 (&pf)[2][2]) __attribute__((always_inline)) {
    // Along a sequence maxima soon stop growing: the sums are rescaled where one of the wavefront's rows has a new reference
    if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0ull) {
      const Two by = both_rows(alpha);
      l_run[0] *= by.x;
      l_run[1] *= by.y;
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        oacc[db][0] *= by.x;
        oacc[db][1] *= by.y;
      }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float l[2] = {0.f, 0.f};
#pragma unroll
      for (int sp = 0; sp < 2; ++sp)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[2 * sp + (e >> 2)][x][e & 3], c2, -(x ? mc.y : mc.x)));
          l[e & 1] += p;
          pf[x][sp][e] = (bf16_t)p;
        }
      l_run[x] += l[0] + l[1];
    }
  };

  if (steps > 0) {
    // A wavefront takes a matrix phase and a vector phase in turn: values of a piece and scores of the next, probabilities of those.  Of the two wavefronts of a SIMD one has the matrix
    // pipe while the other makes probabilities: a barrier after every phase keeps them so, the second half of the wavefronts a phase behind.  With the products of a piece (8 bits: in the
    // vector phase behind them) K of the third piece on and V of the second one on are asked for; they are there at the end of the next vector phase.  (One barrier for two pieces, a phase
    // apart all the same: 3970 clocks a piece where this took 3640, and all eight in step 4180.  Asked for in the vector phase in 16 bits too: 1 % longer; maxima beside the products: 5 %.)
    const bool behind = wave >= kChunkWaves / 2;
    auto tile = [](int step) { return (uint32_t)(step & (kStages - 1)) * kPieceBytes; };
    auto turn = [&]() __attribute__((always_inline)) {
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    f32x4 s[4][2];
    bf16x8 pf[2][2], frag[kAhead];
    u32x4 kr, vr;  // e4m3: on the way to LDS
    look_up(0);
    asm volatile("" : "+v"(qf[0][0]), "+v"(qf[0][1]), "+v"(qf[0][2]), "+v"(qf[0][3]), "+v"(qf[1][0]), "+v"(qf[1][1]), "+v"(qf[1][2]), "+v"(qf[1][3]));  // (waited for here, not in the loop)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const Move m = move_of(i);
      stage(k_base, m, m.ks(), tile(i));
      if (i == 0) stage(v_base, m, m.vs(), kChunkV);
    }
    if constexpr (kE4m3) {
      kr = fetch(k_base, move_of(2));
      vr = fetch(v_base, move_of(1));
    } else {
      move(k_base, move_of(2), tile(2));
      move(v_base, move_of(1), kChunkV + tile(1));
    }
    // what is asked for with piece `step`, made out beside its products
    Move m2, m3;
    uint32_t seen;
    auto prepare = [&](int step) __attribute__((always_inline)) {
      seen = word_at(step);
      m2 = move_of(step + 2);
      m3 = move_of(step + 3);
    };
    auto send = [&](int step) __attribute__((always_inline)) {
      if constexpr (kE4m3) {
        put(kr, m2.ks(), tile(step + 2));
        put(vr, Move{0, 0, word_at(step + 1)}.vs(), kChunkV + tile(step + 1));
        kr = fetch(k_base, m3);
        vr = fetch(v_base, m2);
      }
      if (step + 1 - base == 61) look_up(base + 61);
    };
    auto request = [&](int step) __attribute__((always_inline)) {
      if constexpr (!kE4m3) {
        move(k_base, m3, tile(step + 3));
        move(v_base, m2, kChunkV + tile(step + 2));
      }
    };
    auto sent = [&]() __attribute__((always_inline)) {
      if constexpr (kE4m3) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      else asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    };
    auto nothing = [](int) __attribute__((always_inline)) {};
    if constexpr (!kE4m3) wait_loads();
    __syncthreads();
    if (behind) turn();
    prepare(0);
    if (wave_on) {
      first_operands<true>(keys(0), values(0), frag);
      matrix_phase<true, false>(keys(0), values(0), qf, pf, s, oacc, frag, nothing);
    }
    request(0);
    turn();
    send(0);
    if (wave_on) {
      reference(0, seen, s);
      probabilities(s, pf);
    }
    sent();
#pragma unroll 1
    for (int step = 1; step < steps; ++step) {
      if (wave_on) first_operands<true>(keys(tile(step)), values(0), frag);
      turn();
      if (wave_on) {
        __builtin_amdgcn_s_setprio(1);
        matrix_phase<true, true>(keys(tile(step)), values(tile(step - 1)), qf, pf, s, oacc, frag, [&](int i) __attribute__((always_inline)) {
          if (i == 11) prepare(step);
          if (i == 21) request(step);
        });
        __builtin_amdgcn_s_setprio(0);
      } else {
        prepare(step);
        request(step);
      }
      turn();
      send(step);
      if (wave_on) {
        reference(step, seen, s);
        probabilities(s, pf);
      }
      sent();
    }
    if (wave_on) first_operands<false>(keys(0), values(tile(steps - 1)), frag);
    turn();
    if (wave_on) matrix_phase<false, true>(keys(0), values(tile(steps - 1)), qf, pf, s, oacc, frag, nothing);
    if (!behind) turn();
    wait_loads();
    __syncthreads();  // the tiles are free

    // Tokens of the unit see different keys of a piece, and what one does not see may be an infinity or a NaN, which a probability of zero does not silence.  Such a value
    // leaves its mark in the sums: then the span is gone through again, piece by piece, and where rows of the wavefront see different keys one token at a time, the others'
    // keys as zeros.
    float mark = 0.f;
#pragma unroll
    for (int db = 0; db < 8; ++db)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) mark = fmaf(oacc[db][x][e], 0.f, mark);
    uint32_t* marks = reinterpret_cast<uint32_t*>(smem);
    const bool marked = __builtin_amdgcn_ballot_w64(wave_on && mark != 0.f) != 0ull;
    if (lane == 0) marks[wave] = marked;
    __syncthreads();
    uint32_t any = 0;
#pragma unroll
    for (int w = 0; w < kChunkWaves; ++w) any |= marks[w];
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane((int)any)) {
      clear();
      const Cache& C = arguments().C;
      const ChunkArgs& A = arguments().A;
      const int limit = C.max_pages << C.page_log2, rows = W.nt * C.g, window = A.window;
      const int token[2] = {lane_row(C, A, W, wave, 0).token, lane_row(C, A, W, wave, 1).token};
      const int t_first = div_g(32 * wave, C.g, A.g_magic), t_last = div_g(min(32 * wave + 31, rows - 1), C.g, A.g_magic);
#pragma unroll 1
      for (int step = 0; step < steps; ++step) {
        if (step == 0 || step - base == 64) look_up(step);
        load_q();  // (not kept: the registers are what this loop is short of)
        const Move a = move_of(step);
        stage(k_base, a, a.ks(), 0);
        stage(v_base, a, a.vs(), kChunkV);
        wait_loads();
        __syncthreads();
        if (wave_on) {
          first_operands<true>(keys(0), values(0), frag);
          matrix_phase<true, false>(keys(0), values(0), qf, pf, s, oacc, frag, nothing);
          const int key0 = (first + step) * 64;
          reference(step, a.word, s);
          probabilities(s, pf);
          if (a.word & 16) {
            first_operands<false>(keys(0), values(0), frag);
            matrix_phase<false, true>(keys(0), values(0), qf, pf, s, oacc, frag, nothing);
          } else {
#pragma unroll
            for (int sp = 0; sp < 2; ++sp) {
#pragma unroll 1
              for (int k = t_first; k <= t_last; ++k) {
                const int k_hi = min(W.place + k + 1, limit) - key0, k_lo = (window > 0 ? max(W.place + k + 1 - window, 0) : 0) - key0;
#pragma unroll
                for (int db = 0; db < 8; ++db) {
                  __builtin_amdgcn_sched_barrier(0);  // one product's operands at a time
                  uint32_t at = values(0);
                  asm volatile("" : "+v"(at));
                  bf16x8 v = value_operand(at, sp, db);
#pragma unroll
                  for (int e = 0; e < 8; ++e) {
                    const int key = 32 * sp + 16 * (e >> 2) + (e & 3);  // and 4 part
                    if (4 * part < k_lo - key || 4 * part >= k_hi - key) v[e] = (bf16_t)0.f;
                  }
#pragma unroll
                  for (int x = 0; x < 2; ++x) {
                    const f32x4 add = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, pf[x][sp], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) oacc[db][x][e] += token[x] == k ? add[e] : 0.f;
                  }
                }
              }
            }
          }
        }
        __syncthreads();  // the tiles are overwritten by the next piece
      }
    }
  }
  const float l_all = row_sum(l_run[0], l_run[1]);  // of the first or the second row, as ref

  const Cache& C = arguments().C;
  const ChunkArgs& A = arguments().A;
  const int rows = W.nt * C.g;
  if (!wave_on) return;
  const int lane_b = own_lane(), col = lane_b & 15, quarter = lane_b >> 4;
  if (!P.whole) {
    f32x4* to = reinterpret_cast<f32x4*>(A.part) + ((int64_t)P.slot * kChunkWaves + wave) * 1024 + lane_b;
#pragma unroll
    for (int db = 0; db < 8; ++db)
#pragma unroll
      for (int x = 0; x < 2; ++x) to[64 * (2 * db + x)] = oacc[db][x];
    if ((quarter & 1) == 0) A.part_ml[(int64_t)P.slot * kChunkRows + 32 * wave + 16 * (quarter >> 1) + col] = float2{ref, l_all};
    return;
  }
  const Two total = both_rows(l_all);
  char* own = smem + 32 * wave * kPieceRow;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const LaneRow L = lane_row(C, A, W, wave, x);
    const float l = x ? total.y : total.x, inv = 1.f / l;
    const bool some = l > 0.f || l != l;
    float gate = 0.f;
    uint2 acc[8];
#pragma unroll
    for (int db = 0; db < 8; ++db) acc[db] = uint2{0u, 0u};
    if (A.gate && L.here) {
      gate = A.gate[L.row];
      if (A.o_acc) {
#pragma unroll
        for (int db = 0; db < 8; ++db) acc[db] = *reinterpret_cast<const uint2*>((const bf16_t*)A.o_acc + L.row * kD + 16 * db + 4 * quarter);
      }
    }
#pragma unroll
    for (int db = 0; db < 8; ++db) {
      float o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = some ? oacc[db][x][e] * inv : 0.f;  // an empty row is 0 whatever its values are
      if (A.gate) {
        o[0] = fmaf(gate, o[0], bf16_lo(acc[db].x));
        o[1] = fmaf(gate, o[1], bf16_hi(acc[db].x));
        o[2] = fmaf(gate, o[2], bf16_lo(acc[db].y));
        o[3] = fmaf(gate, o[3], bf16_hi(acc[db].y));
      }
      *reinterpret_cast<uint2*>(own + (16 * x + col) * kPieceRow + (((2 * db + (quarter >> 1)) ^ col) << 4) + 8 * (quarter & 1)) = uint2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
    }
    const float at = x ? both_rows(ref).y : both_rows(ref).x;
    if (quarter == 0 && L.here) A.LSE[L.row] = some ? (finite_reference(at) + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
  }
  wave_sync();
  const int sub = lane_b & 15;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int wr = 4 * i + (lane_b >> 4), rr = 32 * wave + wr;
    if (rr >= rows) break;
    const int t = div_g(rr, C.g, A.g_magic), h = rr - t * C.g;
    *reinterpret_cast<u32x4*>((bf16_t*)A.O + ((int64_t)(W.t0 + t) * C.hq + W.j * C.g + h) * kD + 8 * sub) =
        *reinterpret_cast<const u32x4*>(own + wr * kPieceRow + ((sub ^ (wr & 15)) << 4));
  }
}

// All units' pieces cut into equal parts, one for each workgroup, one after the other, so that all workgroups end together whatever the lengths, which only the device knows.  A workgroup
// finds its first unit by a scan over those of a head.
__device__ __forceinline__ int64_t uniform(int64_t x) {  // a value that all lanes have, in scalar registers
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}
struct State {
  int s, i, j, t0, nt, place;  // the unit
  int64_t q, left;             // where the workgroup begins in it, what is left to be done, in pieces
  int share;                   // what a workgroup does, where that is less than 2^31
};
// Where a unit of this cost is cut if an equal share ends at x: not so near its ends that a part of it would cost more than it is worth.
__device__ __forceinline__ int64_t cut_at(int64_t x, int64_t cost) { return x < kUnitCost + kLeastSpan ? 0 : x > cost - kLeastSpan ? cost : x; }
static_assert(sizeof(State) <= kChunkLds - 2 * kStages * kPieceBytes, "it lies behind the tiles");
template <bool kE4m3>
__global__ void __launch_bounds__(kChunkThreads, 2) k_cache_chunk_even(Args) {
  const Cache& C = arguments().C;
  const ChunkArgs& A = arguments().A;
  extern __shared__ __align__(256) char smem[];
  // XCDs get workgroups in turn, and take an eighth of all pieces each: with eight KV heads one head's, which its L2 then serves
  const int wg = (int)(blockIdx.x & 7) * (A.slots >> 3) + (int)(blockIdx.x >> 3);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = (A.units + kChunkThreads - 1) / kChunkThreads, u0 = threadIdx.x * per, u1 = min(u0 + per, A.units);
  // of the units u0 .. u1 - 1 of a head, `visit` those that there are with their cost
  auto each_unit = [&](auto visit) __attribute__((always_inline)) {
    if (u0 >= u1) return;
    int lo = 0, hi = C.nseq;  // the last sequence that starts at u0 or before
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first_unit(C, A, mid) <= u0) lo = mid;
      else hi = mid;
    }
    int s = lo;
    for (int u = u0; u < u1; ++u) {
      while (s + 1 < C.nseq && first_unit(C, A, s + 1) <= u) ++s;
      const int64_t i = u - first_unit(C, A, s);
      if (i < 0) continue;
      const Unit W = unit_of(C, A, s, (int)i, 0);
      if (W.s >= 0 && !visit(W, (int)i, kUnitCost + pieces_of(C, A, W).y)) return;
    }
  };
  int64_t own = 0;
  Unit head;  // the first of them
  int head_i = 0, head_cost = 0;
  each_unit([&](const Unit& W, int i, int cost) {
    if (own == 0) {
      head = W;
      head_i = i;
      head_cost = cost;
    }
    own += cost;
    return true;
  });
  int64_t upto = own;
  for (int d = 1; d < 64 && d < A.units; d <<= 1) {
    const int64_t x = __shfl_up(upto, d);
    if (lane >= d) upto += x;
  }
  int64_t* sums = reinterpret_cast<int64_t*>(smem);
  if (lane == 63) sums[wave] = A.units < 64 ? 0 : upto;
  if (A.units < 64 && threadIdx.x == A.units - 1) sums[0] = upto;
  __syncthreads();
  int64_t before = upto - own, of_head = 0;
#pragma unroll
  for (int w = 0; w < kChunkWaves; ++w) {
    if (w < wave) before += sums[w];
    of_head += sums[w];
  }
  of_head = uniform(of_head);
  const int64_t total = of_head * C.hkv, share = max((total + A.slots - 1) / A.slots, (int64_t)kLeastShare), start = wg * share;
  if (threadIdx.x == 0) A.joints[wg].parts = 0;
  if (start >= total) return;  // the whole workgroup
  const int j = total < (int64_t)1 << 32 ? (int)((uint32_t)start / (uint32_t)of_head) : (int)(start / of_head);
  const int64_t at = start - j * of_head;
  // Where the workgroup stands lies in LDS behind the tiles, and not in registers that the units want
  State* state = reinterpret_cast<State*>(smem + 2 * kStages * kPieceBytes);
  if (before <= at && at < before + own) {
    int64_t sum = before;
    auto here = [&](const Unit& W, int i, int cost) {
      if (at < sum + cost) {
        *state = State{W.s, i, j, W.t0, W.nt, W.place, at - sum, min(share, total - start), (int)min(share, (int64_t)INT32_MAX)};
        return false;
      }
      sum += cost;
      return true;
    };
    if (here(head, head_i, head_cost)) {
      sum = before;
      each_unit(here);
    }
  }
  __syncthreads();
  for (;;) {
    {
      const Cache& C = arguments().C;
      const ChunkArgs& A = arguments().A;
      const Unit W = {state->s, state->t0, state->nt, state->place, state->j};
      const int64_t q = uniform(state->q), left = uniform(state->left);
      const int n = pieces_of(C, A, W).y;
      const int64_t cost = kUnitCost + n, begin = cut_at(q, cost), end = q + left >= cost ? cost : cut_at(q + left, cost);
      const int wg = (int)(blockIdx.x & 7) * (A.slots >> 3) + (int)(blockIdx.x >> 3);
      Span P;
      P.begin = max((int)begin - kUnitCost, 0);
      P.end = max((int)end - kUnitCost, 0);
      P.whole = begin == 0 && end == cost;
      P.slot = 2 * wg + (begin == 0 ? 1 : 0);
      if (begin == 0 && 0 < end && end < cost && threadIdx.x == 0) {
        // the others' parts: one for each cut of the unit
        A.joints[wg] = Joint{W.t0, W.nt, W.j, 2 + (int)((uint32_t)(cost - kLeastSpan - end) / (uint32_t)state->share), P.slot, 2 * (wg + 1), {0, 0}};
      }
      __syncthreads();  // all have read the state
      if (threadIdx.x == 0) {
        state->left = left - (cost - q);
        state->q = 0;
      }
      if (begin < end) attend_unit<kE4m3>(W, P, smem);
    }
    __syncthreads();  // the LDS is the next unit's
    if (state->left <= 0) return;
    const Cache& C = arguments().C;
    const ChunkArgs& A = arguments().A;
    // the next unit: of the sequence, of the next one that has tokens, of the next head
    int s = __builtin_amdgcn_readfirstlane(state->s), i = __builtin_amdgcn_readfirstlane(state->i) + 1, j = __builtin_amdgcn_readfirstlane(state->j);
    const int c1 = C.cu ? C.cu[s + 1] : s + 1, c0 = C.cu ? C.cu[s] : s;
    if (c0 + (int64_t)i * A.tok >= min(c1, C.T)) {
      int t = c1;
      if (t >= C.T || (C.cu && t >= C.cu[C.nseq])) {
        ++j;
        t = C.cu ? max(C.cu[0], 0) : 0;
      }
      s = C.cu ? find_sequence(C.nseq, t, [&](int x) { return (int64_t)C.cu[x]; }) : t;
      i = 0;
      if (s < 0 || j >= C.hkv) return;  // (starts that are not in order)
    }
    const Unit W = unit_of(C, A, s, i, j);
    __syncthreads();  // all have read the state
    if (threadIdx.x == 0) {
      state->s = s;
      state->i = i;
      state->j = j;
      state->t0 = W.t0;
      state->nt = W.nt;
      state->place = W.place;
    }
    __syncthreads();
  }
}

// The parts of a unit that several workgroups had: a workgroup joins 32 of its rows, a wavefront 32 channels of every second part of them.
__global__ void __launch_bounds__(kChunkJoinThreads) k_cache_chunk_join(Args X) {
  const Cache& C = X.C;
  const ChunkArgs& A = X.A;
  __shared__ __align__(16) char smem[4 * 5 * 64 * 16];
  constexpr int kBatch = 4;
  const int b = (int)(blockIdx.x >> 3), rw = (int)(blockIdx.x & 7);
  const Joint J = A.joints[b];
  const int rows = J.nt * C.g, n = J.parts;
  if (n == 0 || 32 * rw >= rows) return;
  const int lane = threadIdx.x & 63, db = threadIdx.x >> 6 & 3, half = threadIdx.x >> 8, col = lane & 15, quarter = lane >> 4;
  // this lane's rows col and 16 + col; o[2 h + x]: channels 32 db + 16 h + 4 quarter .. of row x
  int64_t row[2];
  bool here[2];
  int rc[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int r = 32 * rw + 16 * x + col;
    here[x] = r < rows;
    rc[x] = min(r, rows - 1);
    const int tt = div_g(rc[x], C.g, A.g_magic);
    row[x] = (int64_t)(J.t0 + tt) * C.hq + J.j * C.g + rc[x] - tt * C.g;
  }
  float top[2] = {-INFINITY, -INFINITY}, total[2] = {0.f, 0.f};
  f32x4 o[4];
#pragma unroll
  for (int a = 0; a < 4; ++a) o[a] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto add = [&](int x, float ref, float sum, const f32x4& first, const f32x4& second) __attribute__((always_inline)) {
    float f0;
    const float mc = new_reference(ref, top[x], f0), f1 = __builtin_amdgcn_exp2f(ref - mc);
    total[x] = fmaf(total[x], f0, f1 * sum);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[x][e] = fmaf(o[x][e], f0, f1 * first[e]);
      o[2 + x][e] = fmaf(o[2 + x][e], f0, f1 * second[e]);
    }
  };
  for (int i0 = half; i0 < n; i0 += 2 * kBatch) {
    float2 ml[kBatch][2];
    f32x4 y[kBatch][4];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int i = min(i0 + 2 * k, n - 1);
      const int64_t at = min(i == 0 ? J.first : J.second + 2 * (i - 1), 2 * kSlots - 1);  // (less in any case, unless starts are not in order)
#pragma unroll
      for (int x = 0; x < 2; ++x) ml[k][x] = A.part_ml[at * kChunkRows + rc[x]];
      const f32x4* from = reinterpret_cast<const f32x4*>(A.part) + (at * kChunkWaves + rw) * 1024 + 256 * db + lane;
#pragma unroll
      for (int a = 0; a < 4; ++a) y[k][a] = from[64 * a];
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (i0 + 2 * k >= n) break;
#pragma unroll
      for (int x = 0; x < 2; ++x) add(x, ml[k][x].x, ml[k][x].y, y[k][x], y[k][2 + x]);
    }
  }
  f32x4* hand = reinterpret_cast<f32x4*>(smem) + db * 5 * 64 + lane;
  if (half == 1) {
    hand[0] = f32x4{top[0], total[0], top[1], total[1]};
#pragma unroll
    for (int a = 0; a < 4; ++a) hand[64 * (1 + a)] = o[a];
  }
  __syncthreads();
  if (half == 0) {
    const f32x4 his = hand[0];
#pragma unroll
    for (int x = 0; x < 2; ++x) add(x, his[2 * x], his[2 * x + 1], hand[64 * (1 + x)], hand[64 * (3 + x)]);
  }
  __syncthreads();
  if (half == 0) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const bool some = total[x] > 0.f || total[x] != total[x];
      const float inv = 1.f / total[x];
      float gate = 0.f;
      if (A.gate && here[x]) gate = A.gate[row[x]];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x4 y = o[2 * h + x];
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = some ? y[e] * inv : 0.f;
        if (A.gate) {
          uint2 z = {0u, 0u};
          if (A.o_acc && here[x]) z = *reinterpret_cast<const uint2*>((const bf16_t*)A.o_acc + row[x] * kD + 32 * db + 16 * h + 4 * quarter);
          y[0] = fmaf(gate, y[0], bf16_lo(z.x));
          y[1] = fmaf(gate, y[1], bf16_hi(z.x));
          y[2] = fmaf(gate, y[2], bf16_lo(z.y));
          y[3] = fmaf(gate, y[3], bf16_hi(z.y));
        }
        *reinterpret_cast<uint2*>(smem + (16 * x + col) * kPieceRow + (((4 * db + 2 * h + (quarter >> 1)) ^ col) << 4) + 8 * (quarter & 1)) =
            uint2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
      }
      if (db == 0 && quarter == 0 && here[x]) A.LSE[row[x]] = some ? (finite_reference(top[x]) + __builtin_amdgcn_logf(total[x])) * 0.6931471805599453f : -INFINITY;
    }
  }
  __syncthreads();
  const int sub = threadIdx.x & 15, wr = (int)(threadIdx.x >> 4), rr = 32 * rw + wr;
  if (rr >= rows) return;
  const int t = div_g(rr, C.g, A.g_magic), h = rr - t * C.g;
  *reinterpret_cast<u32x4*>((bf16_t*)A.O + ((int64_t)(J.t0 + t) * C.hq + J.j * C.g + h) * kD + 8 * sub) =
      *reinterpret_cast<const u32x4*>(smem + wr * kPieceRow + ((sub ^ (wr & 15)) << 4));
}

// ---- host -----------------------------------------------------------------------------------------------------------------------------
struct ChunkCut {
  int tok, slots;
  int64_t units;
  size_t ml, joints, total;  // offsets in the workspace; the sums come first
};
ChunkCut chunk_cut(const nsa_sel_cache_shape* s) {
  ChunkCut c;
  c.tok = kChunkRows / (s->hq / s->hkv);
  c.units = (int64_t)s->n_tokens / c.tok + s->nseq;
  // no more workgroups than there can be shares: what the table, or the window, lets a unit see at most  (16 tokens behind 4080 keys: 22.7 us, with all of them 23.3)
  int64_t pieces = ((int64_t)s->max_pages * s->page + 63) / 64;
  if (window_of(s) > 0 && pieces > (window_of(s) + c.tok) / 64 + 2) pieces = (window_of(s) + c.tok) / 64 + 2;
  const int64_t rows = c.units * s->hkv;  // a unit of a head is a share at least
  static_assert(kUnitCost >= kLeastShare);
  const int64_t shares = rows < kSlots ? (rows * (kUnitCost + pieces) + kLeastShare - 1) / kLeastShare : kSlots;
  c.slots = shares < kSlots ? (int)((shares + 7) & ~(int64_t)7) : kSlots;
  c.ml = (size_t)2 * kSlots * kChunkRows * kD * 4;
  c.joints = c.ml + (size_t)2 * kSlots * kChunkRows * 8;
  c.total = c.joints + kSlots * sizeof(Joint);
  return c;
}
int check_chunk_shape(const nsa_sel_cache_shape* s) {
  const int rc = check_sizes(s, true);
  if (rc) return rc;
  if (s->topk != 0) return NSA_SEL_EINVAL;
  return chunk_cut(s).units < (int64_t)1 << 31 ? NSA_SEL_OK : NSA_SEL_EUNSUPPORTED;
}

}  // namespace
}  // namespace nsa

using namespace nsa;

extern "C" {

int nsa_sel_cache_chunk_workspace_bytes(const nsa_sel_cache_shape* shape, size_t* bytes) {
  const int rc = check_chunk_shape(shape);
  if (rc) return rc;
  if (bytes) *bytes = shape->n_tokens == 0 ? 0 : chunk_cut(shape).total;
  return NSA_SEL_OK;
}

int nsa_sel_cache_attention_chunk(const nsa_sel_cache_shape* shape, const void* Q, const int32_t* cu_seqlens, const int32_t* kv_len,
                                  const int32_t* table, const void* k_pages, const void* v_pages, const float* k_scale, const float* v_scale,
                                  const float* gate, const void* O_acc, void* O, float* LSE, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_chunk_shape(shape);
  if (rc) return rc;
  if (shape->n_tokens == 0) return NSA_SEL_OK;
  rc = check_cache_pointers(shape, k_pages, v_pages, k_scale, v_scale, table, kv_len, cu_seqlens);
  if (rc) return rc;
  if (!tensor(Q) || !tensor(O) || !ints(LSE) || !tensor(O_acc, true) || !ints(gate, true)) return NSA_SEL_EINVAL;
  if ((O_acc && !gate) || O == Q) return NSA_SEL_EINVAL;
  const ChunkCut c = chunk_cut(shape);
  if (!tensor(ws)) return NSA_SEL_EINVAL;
  if (ws_bytes < c.total) return NSA_SEL_EWORKSPACE;
  const Cache C = make_cache(shape, k_pages, v_pages, k_scale, v_scale, table, kv_len, cu_seqlens);
  ChunkArgs A;
  A.Q = Q;
  A.window = window_of(shape);
  A.scale = shape->scale > 0.f ? shape->scale : 0.08838834764831845f;  // 1/sqrt(128)
  A.gate = gate;
  A.o_acc = O_acc;
  A.O = O;
  A.LSE = LSE;
  A.tok = c.tok;
  A.g_magic = C.g == 1 ? 0u : (uint32_t)(((uint64_t)1 << 32) / (uint32_t)C.g + 1);
  A.units = (int32_t)c.units;
  A.slots = c.slots;
  A.part = (float*)ws;
  A.part_ml = (float2*)((char*)ws + c.ml);
  A.joints = (Joint*)((char*)ws + c.joints);
  const bool e4m3 = shape->dtype == NSA_SEL_CACHE_E4M3;
  const auto kern = e4m3 ? k_cache_chunk_even<true> : k_cache_chunk_even<false>;
  static std::atomic<uint64_t> ready[2];
  if (allow_dynamic_lds((const void*)kern, kChunkLds, ready[e4m3]) != hipSuccess) return NSA_SEL_EHIP;
  {
    ProfScope ps(KID_CACHE_CHUNK, (hipStream_t)stream);
    hipLaunchKernelGGL(kern, dim3(c.slots), dim3(kChunkThreads), kChunkLds, (hipStream_t)stream, Args{C, A});
  }
  if (hipGetLastError() != hipSuccess) return NSA_SEL_EHIP;
  ProfScope ps(KID_CACHE_CHUNK_JOIN, (hipStream_t)stream);
  hipLaunchKernelGGL(k_cache_chunk_join, dim3(8 * c.slots), dim3(kChunkJoinThreads), 0, (hipStream_t)stream, Args{C, A});
  return hipGetLastError() == hipSuccess ? NSA_SEL_OK : NSA_SEL_EHIP;
}

}  // extern "C"
