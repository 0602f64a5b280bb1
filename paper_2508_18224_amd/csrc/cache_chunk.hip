// Attention of pieces of prompts over a paged cache (nsa_sel_cache_attention_chunk): every key, or a window, for many new tokens of a sequence at a time.
//
// S = Q K^T, P = softmax(S), O = P V in one pass over the keys with the running maximum and sum of a row.  A key of a KV head is used by g rows of every token that sees
// it, so a workgroup takes 256 rows (256 / g consecutive tokens of a sequence) of a KV head, a unit, and walks the keys in pieces of 64: eight wavefronts of 32 rows, two to a
// SIMD, each with its Q and its output in registers, share a piece's K and V in LDS.  A piece is 32 KB and 8.4 MFLOP, 2048 clocks of the matrix pipes; reading its operands takes the
// LDS as long.
//
// What bounds it is power before the pipes: with random numbers the products of a piece and their operand reads alone take 1.34 us, at 1.7 GHz, which is what a large library product
// reaches too (1.6 PFLOP/s); moving K and V adds 0.14 and the softmax 0.3, as if each were paid for by itself.  2048 new tokens of 32 heads behind 32768 keys (8 KV heads): 1.0 ms,
// 1.13 PFLOP/s.  (64 rows a wavefront, half the operand reads: 1.34 us as well.)
//
// A page of 16 tokens or more is a run of memory, so the eight rows that a wavefront moves of a piece's K and V are always one page's: which one is looked up for 64 pieces
// at a time, a piece a lane.
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
constexpr int kSlots = 256;  // workgroups that share all units' pieces evenly
// What a unit costs beside its pieces, in pieces: its Q, its pages, the first and the last piece, its result, 10 to 12 us for 1.9 of a piece.  (A whole prompt of 8192 tokens: 1300 us
// with none of it counted, 1023 with 5, 1004 with 6, 1013 with 8.)
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
  // parts of units: slot 2 w of workgroup w for the unit that others begin, 2 w + 1 for the one that it begins and others finish
  float* part;       // [slots][8 wavefronts][16][64 lanes][4]: the sums as the lanes hold them
  float2* part_ml;   // [slots][256] (reference, sum)
  struct Joint* joints;
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
  W.place = C.kv_len[s] - n + i0;
  if (W.nt <= 0 || W.t0 < 0) W.s = -1;
  return W;
}
// The pieces that anything of the unit sees: [first, first + count).
__device__ __forceinline__ int2 pieces_of(const Cache& C, const ChunkArgs& A, const Unit& W) {
  const int hi = min(W.place + W.nt, C.max_pages << C.page_log2), lo = A.window > 0 ? max(W.place + 1 - A.window, 0) : 0;
  const int first = lo / 64;
  return {first, max((hi + 63) / 64 - first, 0)};
}

// This lane's operand reads as piece_addresses has them.  Tiles lie at multiples of 256 bytes, so that the reads of a piece differ in bits that are flipped: made anew from
// one address, they take no registers.
struct KeyAddresses {
  uint32_t at;
  __device__ __forceinline__ uint32_t operator[](int s) const { return at ^ (s << 5); }
};
struct ValueAddresses {
  uint32_t at;
  struct Half {
    uint32_t at;
    __device__ __forceinline__ uint32_t operator[](int d) const { return at ^ (d << 6); }
  };
  __device__ __forceinline__ Half operator[](int h) const { return {h ? (at ^ 32) + 8 * kPieceRow : at}; }
};

// threadIdx.x & 63, made anew wherever it is asked for: what derives from it need not be kept.
__device__ __forceinline__ int own_lane() {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  return tid & 63;
}
// This lane's row of a wavefront's 32: token of the unit and row of Q and O.  Lanes past the last row go along with it.
struct LaneRow {
  int r, token;
  int64_t row;
  bool here;
};
__device__ __forceinline__ LaneRow lane_row(const Cache& C, const ChunkArgs& A, const Unit& W, int wave) {
  LaneRow L;
  const int rows = W.nt * C.g;
  L.r = 32 * wave + (own_lane() & 31);
  L.here = L.r < rows;
  const int rc = min(L.r, rows - 1);
  L.token = div_g(rc, C.g, A.g_magic);
  L.row = (int64_t)(W.t0 + L.token) * C.hq + W.j * C.g + (rc - L.token * C.g);
  return L;
}

// What a row's exponents are taken against: its running maximum times scale * log2(e), rounded, and `ref` is that rounded number, so that alpha, what the sums so far are to be
// multiplied by, is exactly 1 while the maximum stays.  With the maximum itself kept, and rounded anew for every piece, alpha would be 1 but for that rounding's error, the same
// for every piece: over 2048 pieces up to 1.7e-4 of the sum.
__device__ __forceinline__ float finite_reference(float ref) { return ref == -INFINITY ? 0.f : ref; }
__device__ __forceinline__ float new_reference(float m, float& ref, float& alpha, float slack) {
  const float now = m > ref + slack ? m : ref, mc = finite_reference(now);
  alpha = __builtin_amdgcn_exp2f(ref - mc);  // exp2(-inf) = 0 on the first piece with a score
  ref = now;
  return mc;
}

// A reference need not be the maximum: probabilities up to 2^kSlack are as good as those up to 1, and the sums are rescaled far more seldom.
constexpr float kSlack = 6.f;

// Maximum of this lane's value and that of the lane 32 on or back, which has the same row.
__device__ __forceinline__ float both_halves_max(float m) {
  const uint32_t x = __builtin_bit_cast(uint32_t, m);
  const auto y = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  const uint32_t low = y[0], high = y[1];  // (by way of integers: a bit cast of an element takes the first one)
  return fmaxf(__builtin_bit_cast(float, low), __builtin_bit_cast(float, high));
}

// Eight rows of a wavefront straight to LDS (see load_to_lds), four a load, the second four 1 KB on on both sides: the instruction's offset counts for both.
__device__ __forceinline__ void load_rows_to_lds(u32x4 b, uint32_t lds, uint32_t off, uint32_t off2) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %3, 0 offen lds\n\tbuffer_load_dwordx4 %2, %3, 0 offen offset:1024 lds"
               :: "s"(lds), "v"(off), "v"(off2), "s"(b) : "memory", "m0");
}

// ---- the products of a matrix phase, in order: 16 of the scores S^T = K Q^T of a piece, 16 of O^T += V^T P^T of the one before.  A wavefront issues in order: operand reads go kAhead
// products ahead.
constexpr int kAhead = 4;
__device__ __forceinline__ bf16x8 phase_operand(const KeyAddresses& k, const ValueAddresses& v, int i) {
  return i < 16 ? lds_read_frag(k[i >> 1] + 32 * (i & 1) * kPieceRow) : value_frag(v, (i - 16) >> 2, (i - 16) & 3);
}
template <bool kScores>
__device__ __forceinline__ void first_operands(const KeyAddresses& k, const ValueAddresses& v, bf16x8 (&frag)[kAhead]) {
#pragma unroll
  for (int i = 0; i < kAhead; ++i) frag[i] = phase_operand(k, v, (kScores ? 0 : 16) + i);
}
template <bool kScores, bool kValues, class Beside>
__device__ __forceinline__ void matrix_phase(const KeyAddresses& k, const ValueAddresses& v, const bf16x8 (&qf)[8], const bf16x8 (&pf)[4], f32x16 (&s)[2],
                                             f32x16 (&oacc)[4], bf16x8 (&frag)[kAhead], Beside beside) {
  constexpr int kFirst = kScores ? 0 : 16, kLast = kValues ? 32 : 16;
  if constexpr (kScores) {
#pragma unroll
    for (int mb = 0; mb < 2; ++mb)
#pragma unroll
      for (int x = 0; x < 16; ++x) s[mb][x] = 0.f;
  }
#pragma unroll
  for (int i = kFirst; i < kLast; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    if (i < 16) s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i % kAhead], qf[i >> 1], s[i & 1], 0, 0, 0);
    else oacc[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i % kAhead], pf[(i - 16) >> 2], oacc[i & 3], 0, 0, 0);
    if (i + kAhead < kLast) frag[i % kAhead] = phase_operand(k, v, i + kAhead);
    beside(i);
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
  const int lane = own_lane(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), qh = lane >> 5;
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
  int first, c_hi, c_lo;           // the first piece; the keys that this lane's row sees
  int least_hi, most_lo;           // what all rows of the wavefront see: rows are in the order of their tokens, the first one sees the fewest later keys
  float c2;
  const char *k_base, *v_base;
  f32x16 oacc[4];
  float ref = -INFINITY, l_run = 0.f;  // see new_reference; the row's sum
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) oacc[db][v] = 0.f;
    ref = -INFINITY;
    l_run = 0.f;
  };
  clear();
  bf16x8 qf[8];
  {
    const Cache& C = arguments().C;
    const ChunkArgs& A = arguments().A;
    const int limit = C.max_pages << C.page_log2, rows = W.nt * C.g;
    first = pieces_of(C, A, W).x + P.begin;
    wave_on = 32 * wave < rows;
    const LaneRow L = lane_row(C, A, W, wave);
    c_hi = min(W.place + L.token + 1, limit);
    c_lo = A.window > 0 ? max(W.place + L.token + 1 - A.window, 0) : 0;
    least_hi = min(W.place + div_g(min(32 * wave, rows - 1), C.g, A.g_magic) + 1, limit);
    most_lo = A.window > 0 ? max(W.place + div_g(min(32 * wave + 31, rows - 1), C.g, A.g_magic) + 1 - A.window, 0) : 0;
    c2 = A.scale * 1.4426950408889634f;
    k_base = C.k;
    v_base = C.v;
    const bf16_t* src = (const bf16_t*)A.Q + L.row * kD + 8 * qh;
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(src + 16 * s);
  }
  const int v_row = ((lane & 15) >> 2) + 4 * qh;
  const uint32_t k_at = lds_address(smem) + (lane & 31) * kPieceRow + ((qh ^ row_turn(lane & 31)) << 4);
  const uint32_t v_at = lds_address(smem + kChunkV) + v_row * kPieceRow + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ row_turn(v_row)) << 4) + 8 * (lane & 1);
  auto keys = [&](uint32_t off) __attribute__((always_inline)) { return KeyAddresses{k_at + off}; };
  auto values = [&](uint32_t off) __attribute__((always_inline)) { return ValueAddresses{v_at + off}; };

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
  const uint32_t move_off = (lane >> 4) * kPieceRow + (((lane & 15) ^ row_turn(8 * wave + (lane >> 4))) << 4), move_off2 = move_off ^ 16;
  auto move = [&](const char* base, const Move& m, uint32_t lds_off) __attribute__((always_inline)) {
    const uint64_t at = (uint64_t)m.from(base);
    load_rows_to_lds(u32x4{(uint32_t)at, (uint32_t)(at >> 32), m.bytes(), 0x00020000u}, lds_rows + lds_off, move_off, move_off2);
  };
  // e4m3: one load of eight rows into registers, to be written to LDS as bf16
  auto fetch = [&](const char* base, const Move& m) __attribute__((always_inline)) {
    return __builtin_amdgcn_raw_buffer_load_b128(buffer_of(m.from(base), m.bytes()), lane * 16, 0, 0);
  };
  const int put_row = 8 * wave + (lane >> 3);
  const uint32_t put_at = lds_address(smem) + put_row * kPieceRow + (((2 * (lane & 7)) ^ row_turn(put_row)) << 4);
  auto put = [&](u32x4 x, float scale, uint32_t lds_off) __attribute__((always_inline)) {
    const uint32_t at = put_at + lds_off;
    lds_write_16(at, eight_bf16(x[0], x[1], scale));
    lds_write_16(at ^ 16, eight_bf16(x[2], x[3], scale));
  };
  // a tile of K or V at once, in front of the main loop and in the simple one
  auto stage = [&](const char* base, const Move& m, float scale, uint32_t lds_off) __attribute__((always_inline)) {
    if constexpr (kE4m3) put(fetch(base, m), scale, lds_off);
    else move(base, m, lds_off);
  };

  // Scores -> what their exponents are taken against: keys that this lane's row does not see become -inf, the row's maximum joins the running one.
  float alpha, mc;
  auto reference = [&](int step, uint32_t word, float slack, f32x16 (&s)[2]) __attribute__((always_inline)) {
    if (!(word & 16)) {
      const int key0 = (first + step) * 64, lim = c_hi - key0 - 4 * qh, lo = c_lo - key0 - 4 * qh;
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          const int key = 32 * mb + 8 * (v >> 2) + (v & 3);  // and 4 qh
          const bool shown = word >> (2 * mb + (v >> 3)) & 1;
          if (key >= (shown ? lim : 0) || key < lo) s[mb][v] = -INFINITY;
        }
    }
    float m[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      m[x] = fmaxf(s[x >> 1][8 * (x & 1)], s[x >> 1][8 * (x & 1) + 1]);
#pragma unroll
      for (int v = 2; v < 8; v += 2) m[x] = fmaxf(fmaxf(m[x], s[x >> 1][8 * (x & 1) + v]), s[x >> 1][8 * (x & 1) + v + 1]);
    }
    mc = new_reference(both_halves_max(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]))) * c2, ref, alpha, slack);
  };
  // Scores -> probabilities as the operands of the four contraction steps of P V; l_run is of this lane's keys.
  auto probabilities = [&](const f32x16 (&s)[2], bf16x8 (&pf)[4]) __attribute__((always_inline)) {
    float l[2] = {0.f, 0.f};
#pragma unroll
    for (int sp = 0; sp < 4; ++sp)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[sp >> 1][8 * (sp & 1) + e], c2, -mc));
        l[e & 1] += p;
        pf[sp][e] = (bf16_t)p;
      }
    l_run = fmaf(l_run, alpha, l[0] + l[1]);
    // Along a sequence maxima soon stop growing: the sums are rescaled where one of the wavefront's rows has a new one
    if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0ull) {
#pragma unroll
      for (int db = 0; db < 4; ++db) oacc[db] *= alpha;
    }
  };

  if (steps > 0) {
    // A wavefront takes a matrix phase and a vector phase in turn: values of a piece and scores of the next, probabilities of those.  Of the two wavefronts of a SIMD one has the matrix
    // pipe while the other makes probabilities: a barrier after every phase keeps them so, the second half of the wavefronts a phase behind.  In the vector phase of a piece K of the
    // third piece on and V of the second one on are asked for; they are there at the end of the next one.  (One barrier for two pieces, a phase apart all the same: 3970 clocks a piece
    // against 3640, and all eight in step 4180.)
    const bool behind = wave >= kChunkWaves / 2;
    auto tile = [](int step) { return (uint32_t)(step & (kStages - 1)) * kPieceBytes; };
    auto turn = [&]() __attribute__((always_inline)) {
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    f32x16 s[2];
    bf16x8 pf[4], frag[kAhead];
    u32x4 kr, vr;  // e4m3: on the way to LDS
    look_up(0);
    await_rows(qf);
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
    // what is asked for in the vector phase of `step`, made out beside the products in front of it
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
      } else {
        move(k_base, m3, tile(step + 3));
        move(v_base, m2, kChunkV + tile(step + 2));
      }
      if (step + 1 - base == 61) look_up(base + 61);
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
    turn();
    send(0);
    if (wave_on) {
      reference(0, seen, kSlack, s);
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
          if (i == 15) prepare(step);
        });
        __builtin_amdgcn_s_setprio(0);
      } else {
        prepare(step);
      }
      turn();
      send(step);
      if (wave_on) {
        reference(step, seen, kSlack, s);
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
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) mark = fmaf(oacc[db][v], 0.f, mark);
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
      const int token = lane_row(C, A, W, wave).token;
      const int t_first = div_g(32 * wave, C.g, A.g_magic), t_last = div_g(min(32 * wave + 31, rows - 1), C.g, A.g_magic);
#pragma unroll 1
      for (int step = 0; step < steps; ++step) {
        if (step == 0 || step - base == 64) look_up(step);
        const Move a = move_of(step);
        stage(k_base, a, a.ks(), 0);
        stage(v_base, a, a.vs(), kChunkV);
        wait_loads();
        __syncthreads();
        if (wave_on) {
          first_operands<true>(keys(0), values(0), frag);
          matrix_phase<true, false>(keys(0), values(0), qf, pf, s, oacc, frag, nothing);
          const int key0 = (first + step) * 64;
          reference(step, a.word, 0.f, s);
          probabilities(s, pf);
          if (a.word & 16) {
            first_operands<false>(keys(0), values(0), frag);
            matrix_phase<false, true>(keys(0), values(0), qf, pf, s, oacc, frag, nothing);
          } else {
#pragma unroll
            for (int sp = 0; sp < 4; ++sp) {
#pragma unroll 1
              for (int k = t_first; k <= t_last; ++k) {
                const int k_hi = min(W.place + k + 1, limit) - key0, k_lo = (window > 0 ? max(W.place + k + 1 - window, 0) : 0) - key0;
#pragma unroll
                for (int db = 0; db < 4; ++db) {
                  __builtin_amdgcn_sched_barrier(0);  // one product's operands at a time
                  ValueAddresses at = values(0);
                  asm volatile("" : "+v"(at.at));
                  bf16x8 x = value_frag(at, sp, db);
#pragma unroll
                  for (int e = 0; e < 8; ++e) {
                    const int key = 16 * sp + 8 * (e >> 2) + (e & 3);  // and 4 qh
                    if (4 * qh < k_lo - key || 4 * qh >= k_hi - key) x[e] = (bf16_t)0.f;
                  }
                  f32x16 add;
#pragma unroll
                  for (int v = 0; v < 16; ++v) add[v] = 0.f;
                  add = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, pf[sp], add, 0, 0, 0);
#pragma unroll
                  for (int v = 0; v < 16; ++v) oacc[db][v] += token == k ? add[v] : 0.f;
                }
              }
            }
          }
        }
        __syncthreads();  // the tiles are overwritten by the next piece
      }
    }
  }
  l_run += __shfl_xor(l_run, 32);

  const Cache& C = arguments().C;
  const ChunkArgs& A = arguments().A;
  const int rows = W.nt * C.g;
  if (!wave_on) return;
  const LaneRow L = lane_row(C, A, W, wave);
  const int lane_b = own_lane(), col = lane_b & 31, half = lane_b >> 5;
  if (!P.whole) {
    {
      f32x4* to = reinterpret_cast<f32x4*>(A.part) + ((int64_t)P.slot * kChunkWaves + wave) * 1024 + lane_b;
#pragma unroll
      for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int a = 0; a < 4; ++a) to[64 * (4 * db + a)] = f32x4{oacc[db][4 * a], oacc[db][4 * a + 1], oacc[db][4 * a + 2], oacc[db][4 * a + 3]};
      if (half == 0) A.part_ml[(int64_t)P.slot * kChunkRows + L.r] = float2{ref, l_run};
    }
    return;
  }
  const bool some = l_run > 0.f || l_run != l_run;
  const float inv = 1.f / l_run;
  float gate = 0.f;
  uint2 acc[16];
#pragma unroll
  for (int x = 0; x < 16; ++x) acc[x] = uint2{0u, 0u};
  if (A.gate && L.here) {
    gate = A.gate[L.row];
    if (A.o_acc) {
#pragma unroll
      for (int x = 0; x < 16; ++x) acc[x] = *reinterpret_cast<const uint2*>((const bf16_t*)A.o_acc + L.row * kD + 8 * x + 4 * half);
    }
  }
  char* own = smem + 32 * wave * kPieceRow;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      float o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = some ? oacc[db][4 * a + e] * inv : 0.f;  // an empty row is 0 whatever its values are
      if (A.gate) {
        const uint2 x = acc[4 * db + a];
        o[0] = fmaf(gate, o[0], bf16_lo(x.x));
        o[1] = fmaf(gate, o[1], bf16_hi(x.x));
        o[2] = fmaf(gate, o[2], bf16_lo(x.y));
        o[3] = fmaf(gate, o[3], bf16_hi(x.y));
      }
      *reinterpret_cast<uint2*>(own + col * kPieceRow + (((4 * db + a) ^ (col & 15)) << 4) + 8 * half) = uint2{pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3])};
    }
  if (half == 0 && L.here) A.LSE[L.row] = some ? (finite_reference(ref) + __builtin_amdgcn_logf(l_run)) * 0.6931471805599453f : -INFINITY;
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

// All units' pieces cut into kSlots equal parts, one after the other, so that all workgroups end together whatever the lengths, which only the device knows.  A workgroup
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
  const int wg = (int)(blockIdx.x & 7) * (kSlots / 8) + (int)(blockIdx.x >> 3);
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
  const int64_t total = of_head * C.hkv, share = max((total + kSlots - 1) / kSlots, (int64_t)kLeastShare), start = wg * share;
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
      const int wg = (int)(blockIdx.x & 7) * (kSlots / 8) + (int)(blockIdx.x >> 3);
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
  __shared__ __align__(16) char smem[4 * 18 * 64 * 4];
  constexpr int kBatch = 4;
  const int b = (int)(blockIdx.x >> 3), rw = (int)(blockIdx.x & 7);
  const Joint J = A.joints[b];
  const int rows = J.nt * C.g, n = J.parts;
  if (n == 0 || 32 * rw >= rows) return;
  const int lane = threadIdx.x & 63, db = threadIdx.x >> 6 & 3, half = threadIdx.x >> 8, col = lane & 31, qh = lane >> 5;
  const int r = 32 * rw + col, rc = min(r, rows - 1), tt = div_g(rc, C.g, A.g_magic), hh = rc - tt * C.g;
  float top = -INFINITY, total = 0.f;
  f32x4 o[4];
#pragma unroll
  for (int a = 0; a < 4; ++a) o[a] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int i0 = half; i0 < n; i0 += 2 * kBatch) {
    float2 x[kBatch];
    f32x4 y[kBatch][4];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int i = min(i0 + 2 * k, n - 1);
      const int64_t at = min(i == 0 ? J.first : J.second + 2 * (i - 1), 2 * kSlots - 1);  // (less in any case, unless starts are not in order)
      x[k] = A.part_ml[at * kChunkRows + rc];
      if (i0 + 2 * k >= n) x[k] = float2{-INFINITY, 0.f};
      const f32x4* from = reinterpret_cast<const f32x4*>(A.part) + (at * kChunkWaves + rw) * 1024 + 256 * db + lane;
#pragma unroll
      for (int a = 0; a < 4; ++a) y[k][a] = from[64 * a];
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (i0 + 2 * k >= n) break;
      float f0;
      const float mc = new_reference(x[k].x, top, f0, 0.f), f1 = __builtin_amdgcn_exp2f(x[k].x - mc);
      total = fmaf(total, f0, f1 * x[k].y);
#pragma unroll
      for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[a][e] = fmaf(o[a][e], f0, f1 * y[k][a][e]);
    }
  }
  float* hand = reinterpret_cast<float*>(smem) + db * 18 * 64 + lane;
  if (half == 1) {
    hand[0] = top;
    hand[64] = total;
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int e = 0; e < 4; ++e) hand[64 * (2 + 4 * a + e)] = o[a][e];
  }
  __syncthreads();
  if (half == 0) {
    float f0;
    const float his = hand[0], mc = new_reference(his, top, f0, 0.f), f1 = __builtin_amdgcn_exp2f(his - mc);
    total = fmaf(total, f0, f1 * hand[64]);
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[a][e] = fmaf(o[a][e], f0, f1 * hand[64 * (2 + 4 * a + e)]);
  }
  __syncthreads();
  if (half == 0) {
    const bool some = total > 0.f || total != total, here = r < rows;
    const float inv = 1.f / total;
    const int64_t row = (int64_t)(J.t0 + tt) * C.hq + J.j * C.g + hh;
    float gate = 0.f;
    if (A.gate && here) gate = A.gate[row];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
#pragma unroll
      for (int e = 0; e < 4; ++e) o[a][e] = some ? o[a][e] * inv : 0.f;
      if (A.gate) {
        uint2 x = {0u, 0u};
        if (A.o_acc && here) x = *reinterpret_cast<const uint2*>((const bf16_t*)A.o_acc + row * kD + 32 * db + 8 * a + 4 * qh);
        o[a][0] = fmaf(gate, o[a][0], bf16_lo(x.x));
        o[a][1] = fmaf(gate, o[a][1], bf16_hi(x.x));
        o[a][2] = fmaf(gate, o[a][2], bf16_lo(x.y));
        o[a][3] = fmaf(gate, o[a][3], bf16_hi(x.y));
      }
      *reinterpret_cast<uint2*>(smem + col * kPieceRow + (((4 * db + a) ^ (col & 15)) << 4) + 8 * qh) = uint2{pack_bf16x2(o[a][0], o[a][1]), pack_bf16x2(o[a][2], o[a][3])};
    }
    if (db == 0 && qh == 0 && here) A.LSE[row] = some ? (finite_reference(top) + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
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
  int tok;
  int64_t units;
  size_t ml, joints, total;  // offsets in the workspace; the sums come first
};
ChunkCut chunk_cut(const nsa_sel_cache_shape* s) {
  ChunkCut c;
  c.tok = kChunkRows / (s->hq / s->hkv);
  c.units = (int64_t)s->n_tokens / c.tok + s->nseq;
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
  A.part = (float*)ws;
  A.part_ml = (float2*)((char*)ws + c.ml);
  A.joints = (Joint*)((char*)ws + c.joints);
  const bool e4m3 = shape->dtype == NSA_SEL_CACHE_E4M3;
  const auto kern = e4m3 ? k_cache_chunk_even<true> : k_cache_chunk_even<false>;
  static std::atomic<uint64_t> ready[2];
  if (allow_dynamic_lds((const void*)kern, kChunkLds, ready[e4m3]) != hipSuccess) return NSA_SEL_EHIP;
  {
    ProfScope ps(KID_CACHE_CHUNK, (hipStream_t)stream);
    hipLaunchKernelGGL(kern, dim3(kSlots), dim3(kChunkThreads), kChunkLds, (hipStream_t)stream, Args{C, A});
  }
  if (hipGetLastError() != hipSuccess) return NSA_SEL_EHIP;
  ProfScope ps(KID_CACHE_CHUNK_JOIN, (hipStream_t)stream);
  hipLaunchKernelGGL(k_cache_chunk_join, dim3(8 * kSlots), dim3(kChunkJoinThreads), 0, (hipStream_t)stream, Args{C, A});
  return hipGetLastError() == hipSuccess ? NSA_SEL_OK : NSA_SEL_EHIP;
}

}  // extern "C"
