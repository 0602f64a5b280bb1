// Attention of pieces of prompts over a paged cache (nsa_sel_cache_attention_chunk): every key, or a window, for many new tokens of a sequence at a time.
//
// S = Q K^T, P = softmax(S), O = P V in one pass over the keys with the running maximum and sum of a row.  A key of a KV head is used by g rows of every token that sees
// it, so a workgroup takes 256 rows (256 / g consecutive tokens of a sequence) of a KV head and walks the keys in pieces of 64: eight wavefronts of 32 rows, two to a
// SIMD, each with its Q and its output in registers, share a piece's K and V in LDS.  A piece is 32 KB and 8.4 MFLOP: bound by the matrix pipe.  The products are those of dense_piece.h.
//
// A page of 16 tokens or more is a run of memory, so the eight rows that a wavefront moves of a piece's K and V are always one page's: which one is looked up for 64 pieces
// at a time, a piece a lane.  Three tiles of K and of V: a piece is requested two steps before it is used.
//
// Probabilities are rounded to bf16 for their product, as in the prompt's own attention (see new_maximum in dense_piece.h: the largest one is exact); the sums they are
// divided by are not.
#include "cache_checks.h"
#include "dense_piece.h"

namespace nsa {
namespace {

constexpr int kChunkWaves = 8, kChunkRows = 32 * kChunkWaves, kChunkThreads = 64 * kChunkWaves;
constexpr int kStages = 3;
constexpr int kChunkV = kStages * kPieceBytes, kChunkLds = 2 * kStages * kPieceBytes + 64;
constexpr int kSlots = 256;  // workgroups that share all units' pieces evenly
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
  // parts of units: slot 2 w of workgroup w for the unit it begins in the middle of, 2 w + 1 for the one that it leaves unfinished
  float* part;       // [slots][8 wavefronts][16][64 lanes][4]: the sums as the lanes hold them
  float2* part_ml;   // [slots][256] (reference, sum)
  int4* whole;       // [hkv][units]: first slot, second slot, number of parts
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
__device__ __forceinline__ float new_reference(float m, float& ref, float& alpha) {
  const float now = fmaxf(ref, m), mc = finite_reference(now);
  alpha = __builtin_amdgcn_exp2f(ref - mc);  // exp2(-inf) = 0 on the first piece with a score
  ref = now;
  return mc;
}

// The part [begin, end) of a unit's pieces that a workgroup takes; if that is not all of them the sums go to slot `slot`.
struct Span {
  int begin, end, slot;
  bool whole;
};

template <bool kE4m3>
__device__ __forceinline__ void attend_unit(const Cache& C, const ChunkArgs& A, Unit W, Span P, char* smem) {
  const int lane = own_lane(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), qh = lane >> 5;
  // the same in every lane, and said so: the buffers below are scalar
  W.s = __builtin_amdgcn_readfirstlane(W.s);
  W.t0 = __builtin_amdgcn_readfirstlane(W.t0);
  W.nt = __builtin_amdgcn_readfirstlane(W.nt);
  W.place = __builtin_amdgcn_readfirstlane(W.place);
  W.j = __builtin_amdgcn_readfirstlane(W.j);
  P.begin = __builtin_amdgcn_readfirstlane(P.begin);
  P.end = __builtin_amdgcn_readfirstlane(P.end);
  const int limit = C.max_pages << C.page_log2;
  const int first = pieces_of(C, A, W).x + P.begin, steps = P.end - P.begin;
  const int hi = min(W.place + W.nt, limit);
  const int rows = W.nt * C.g;
  const bool wave_on = 32 * wave < rows;  // idle wavefronts still move K and V
  // the keys that this lane's row sees
  int c_hi, c_lo;
  const float c2 = A.scale * 1.4426950408889634f;

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
    const LaneRow L = lane_row(C, A, W, wave);
    c_hi = min(W.place + L.token + 1, limit);
    c_lo = A.window > 0 ? max(W.place + L.token + 1 - A.window, 0) : 0;
    const bf16_t* src = (const bf16_t*)A.Q + L.row * kD + 8 * qh;
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(src + 16 * s);
  }
  const int v_row = ((lane & 15) >> 2) + 4 * qh;
  const uint32_t k_at = lds_address(smem) + (lane & 31) * kPieceRow + ((qh ^ row_turn(lane & 31)) << 4);
  const uint32_t v_at = lds_address(smem + kChunkV) + v_row * kPieceRow + (((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ row_turn(v_row)) << 4) + 8 * (lane & 1);
  auto keys = [&](int off) __attribute__((always_inline)) { return KeyAddresses{k_at + off}; };
  auto values = [&](int off) __attribute__((always_inline)) { return ValueAddresses{v_at + off}; };

  // ---- pages: lane l knows those of step i0 + l, whose four 16-token groups may each have another one; this wavefront moves rows 8 wave.. of a piece
  int page_of_step = -1;       // this wavefront's page
  uint32_t word_of_step = 0;   // bits 0-3: groups that have a page; 4-7: rows to be moved; 8-15, 16-23: exponents of the page's scales
  auto look_up = [&](int i0) __attribute__((always_inline)) {
    const int step = i0 + lane, key = (first + step) * 64, own = wave >> 1;
    page_of_step = -1;
    word_of_step = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int p = step < steps ? page_of(C, W.s, key + 16 * q) : -1;
      word_of_step |= p >= 0 ? 1u << q : 0u;
      if (q == own) page_of_step = p;
    }
    if (page_of_step >= 0) {
      word_of_step |= (uint32_t)min(max(hi - (key + 8 * wave), 0), 8) << 4;
      if constexpr (kE4m3) {
        const int64_t head = (int64_t)page_of_step * C.hkv + W.j;
        word_of_step |= (__builtin_bit_cast(uint32_t, C.ks[head]) >> 23 & 255) << 8 | (__builtin_bit_cast(uint32_t, C.vs[head]) >> 23 & 255) << 16;
      }
    }
  };
  struct Move {
    int64_t row;
    uint32_t word;
    __device__ __forceinline__ int rows() const { return word >> 4 & 15; }
    __device__ __forceinline__ int seen() const { return word & 15; }
    __device__ __forceinline__ float ks() const { return __builtin_bit_cast(float, (word >> 8 & 255) << 23); }
    __device__ __forceinline__ float vs() const { return __builtin_bit_cast(float, (word >> 16 & 255) << 23); }
  };
  auto move_of = [&](int step) __attribute__((always_inline)) {
    if ((step & 63) == 0) look_up(step);
    const int page = max(__builtin_amdgcn_readlane(page_of_step, step & 63), 0);
    Move m;
    m.row = (((int64_t)page * C.hkv + W.j) << C.page_log2) + (((first + step) * 64 + 8 * wave) & ((1 << C.page_log2) - 1));
    m.word = (uint32_t)__builtin_amdgcn_readlane((int)word_of_step, step & 63);
    return m;
  };
  // bf16: two loads of four rows, straight to LDS, lane l the place l % 16 of its row
  const int move_turn = row_turn(8 * wave + (lane >> 4));
  const uint32_t move_off = (lane >> 4) * kPieceRow + (((lane & 15) ^ move_turn) << 4);
  auto move = [&](const char* base, const Move& m, int lds_off, int x) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t b = buffer_of(base + m.row * kPieceRow, (uint32_t)m.rows() * kPieceRow);
    load_to_lds(b, lds_address(smem) + lds_off + (8 * wave + 4 * x) * kPieceRow, (x ? move_off ^ 16 : move_off) + 4 * x * kPieceRow);
  };
  // e4m3: one load of eight rows into registers, a step before they are written to LDS as bf16
  auto fetch = [&](const char* base, const Move& m) __attribute__((always_inline)) {
    return __builtin_amdgcn_raw_buffer_load_b128(buffer_of(base + m.row * kD, (uint32_t)m.rows() * kD), lane * 16, 0, 0);
  };
  const int put_row = 8 * wave + (lane >> 3);
  const uint32_t put_at = lds_address(smem) + put_row * kPieceRow + (((2 * (lane & 7)) ^ row_turn(put_row)) << 4);
  auto put = [&](u32x4 x, float scale, int lds_off) __attribute__((always_inline)) {
    lds_write_16(put_at + lds_off, eight_bf16(x[0], x[1], scale));
    lds_write_16((put_at ^ 16) + lds_off, eight_bf16(x[2], x[3], scale));
  };
  // a whole tile of K or V at once, for the simple loop below and in front of the main one
  auto stage = [&](const char* base, const Move& m, float scale, int lds_off) __attribute__((always_inline)) {
    if constexpr (kE4m3) {
      put(fetch(base, m), scale, lds_off);
    } else {
      move(base, m, lds_off, 0);
      move(base, m, lds_off, 1);
    }
  };
  auto tile = [](int step) { return (step % kStages) * kPieceBytes; };

  // keys of the piece of step `step` that this lane's row does not see become -inf; the row's maximum over this lane's keys is m
  auto hide = [&](int step, int seen, f32x16 (&cur)[2], float m) __attribute__((always_inline)) {
    const int key0 = (first + step) * 64, lim = c_hi - key0, lo = c_lo - key0;
    if (__builtin_amdgcn_ballot_w64(lim < 64 || lo > 0) != 0ull) m = mask_scores(cur, lo, lim, qh);
    if (seen != 15) {  // groups of keys without a page
      m = -INFINITY;
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          if (!((seen >> (2 * mb + (v >> 3))) & 1)) cur[mb][v] = -INFINITY;
          m = fmaxf(m, cur[mb][v]);
        }
    }
    return row_max(m);
  };

  if (steps > 0) {
    f32x16 even[2], odd[2];
    Move m2, m1;   // of the steps whose K and V are requested next
    int seen0, seen1;
    u32x4 kr, vr;
    float m = -INFINITY;
    await_rows(qf);
    {
      const Move a = move_of(0);
      stage(C.k, a, a.ks(), tile(0));
      stage(C.v, a, a.vs(), kChunkV + tile(0));
      const Move b = move_of(1);
      stage(C.k, b, b.ks(), tile(1));
      const Move c = move_of(2);
      if constexpr (kE4m3) {
        kr = fetch(C.k, c);
        vr = fetch(C.v, b);
      } else {
        stage(C.v, b, 1.f, kChunkV + tile(1));
        stage(C.k, c, 1.f, tile(2));
      }
      seen0 = a.seen();
      seen1 = b.seen();
      m1 = b;
      m2 = c;
    }
    if constexpr (!kE4m3) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    __syncthreads();  // the first piece and the second one's K are there
    if (wave_on) {
      piece_scores(keys(0), qf, even);
      m = max_scores(even);
    }
    // Every step but the last: this piece's values beside the next one's scores.  In flight meanwhile: V of the next piece and K of the one after it, sent off a step ago;
    // now V of the piece after next and K of the one behind that, into the tiles that the last step has read.
    auto piece = [&](int step, f32x16 (&cur)[2], f32x16 (&next)[2]) __attribute__((always_inline)) {
      const Move m3 = move_of(step + 3);
      if constexpr (kE4m3) {
        put(kr, m2.ks(), tile(step + 2));
        put(vr, m1.vs(), kChunkV + tile(step + 1));
        kr = fetch(C.k, m3);
        vr = fetch(C.v, m2);
      }
      const int ko = tile(step + 1), vo = tile(step), k_to = tile(step + 3), v_to = kChunkV + tile(step + 2);
      if (wave_on) {
        float alpha;
        const float mc = new_reference(hide(step, seen0, cur, m) * c2, ref, alpha);
        // Along a sequence maxima soon stop growing: the sums are rescaled where one of the wavefront's rows has a new one
        if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0ull) {
#pragma unroll
          for (int db = 0; db < 4; ++db) oacc[db] *= alpha;
        }
        m = piece_values_and_next_scores<false>(keys(ko), values(vo), qf, c2, mc, alpha, cur, next, l_run, oacc, [&](int i) __attribute__((always_inline)) {
          if constexpr (!kE4m3) {
            if (i < 2) move(C.v, m2, v_to, i);
            else if (i < 4) move(C.k, m3, k_to, i - 2);
          }
        });
      } else if constexpr (!kE4m3) {
        stage(C.v, m2, 1.f, v_to);
        stage(C.k, m3, 1.f, k_to);
      }
      seen0 = seen1;
      seen1 = m2.seen();
      m1 = m2;
      m2 = m3;
      if constexpr (!kE4m3) asm volatile("s_waitcnt vmcnt(4)" ::: "memory");  // what was sent off a step ago
      __syncthreads();  // this piece has been read, the next one is there
    };
    for (int step = 0; step + 1 < steps; step += 2) {
      piece(step, even, odd);
      if (step + 2 < steps) {
        piece(step + 1, odd, even);
      } else {
#pragma unroll
        for (int mb = 0; mb < 2; ++mb) even[mb] = odd[mb];
      }
    }
    if (wave_on) {
      float alpha;
      const float mc = new_reference(hide(steps - 1, seen0, even, m) * c2, ref, alpha);
      piece_values(values(tile(steps - 1)), c2, mc, alpha, even, l_run, oacc);
    }
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
      const int token = lane_row(C, A, W, wave).token;
      const int t_first = div_g(32 * wave, C.g, A.g_magic), t_last = div_g(min(32 * wave + 31, rows - 1), C.g, A.g_magic);
#pragma unroll 1
      for (int step = 0; step < steps; ++step) {
        const Move a = move_of(step);
        stage(C.k, a, a.ks(), 0);
        stage(C.v, a, a.vs(), kChunkV);
        wait_loads();
        __syncthreads();
        if (wave_on) {
          piece_scores(keys(0), qf, even);
          const int key0 = (first + step) * 64;
          const bool border = __builtin_amdgcn_ballot_w64(c_hi - key0 < 64 || c_lo - key0 > 0) != 0ull;
          float alpha;
          const float mc = new_reference(hide(step, a.seen(), even, max_scores(even)) * c2, ref, alpha);
          if (!border) {
            piece_values(values(0), c2, mc, alpha, even, l_run, oacc);
          } else {
            float l = 0.f;
#pragma unroll
            for (int db = 0; db < 4; ++db) oacc[db] *= alpha;
#pragma unroll
            for (int sp = 0; sp < 4; ++sp) {
              const bf16x8 pf = piece_probabilities(even, sp, c2, mc, l);
#pragma unroll 1
              for (int k = t_first; k <= t_last; ++k) {
                const int k_hi = min(W.place + k + 1, limit) - key0, k_lo = (A.window > 0 ? max(W.place + k + 1 - A.window, 0) : 0) - key0;
#pragma unroll
                for (int db = 0; db < 4; ++db) {
                  __builtin_amdgcn_sched_barrier(0);  // one product's operands at a time
                  ValueAddresses at = values(0);
                  asm volatile("" : "+v"(at.at));
                  bf16x8 a = value_frag(at, sp, db);
#pragma unroll
                  for (int e = 0; e < 8; ++e) {
                    const int key = 16 * sp + 8 * (e >> 2) + (e & 3);  // and 4 qh
                    if (4 * qh < k_lo - key || 4 * qh >= k_hi - key) a[e] = (bf16_t)0.f;
                  }
                  f32x16 add;
#pragma unroll
                  for (int v = 0; v < 16; ++v) add[v] = 0.f;
                  add = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pf, add, 0, 0, 0);
#pragma unroll
                  for (int v = 0; v < 16; ++v) oacc[db][v] += token == k ? add[v] : 0.f;
                }
              }
            }
            l_run = fmaf(l_run, alpha, l + __shfl_xor(l, 32));
          }
        }
        __syncthreads();  // the tiles are overwritten by the next piece
      }
    }
  }

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
  if (A.gate && L.here) gate = A.gate[L.row];
  char* own = smem + 32 * wave * kPieceRow;
#pragma unroll
  for (int db = 0; db < 4; ++db)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      float o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = some ? oacc[db][4 * a + e] * inv : 0.f;  // an empty row is 0 whatever its values are
      if (A.gate) {
        uint2 x = {0u, 0u};
        if (A.o_acc && L.here) x = *reinterpret_cast<const uint2*>((const bf16_t*)A.o_acc + L.row * kD + 32 * db + 8 * a + 4 * half);
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
  int s, i, j, first;      // the unit; whether it is the workgroup's first
  int64_t q, left, share;  // pieces of it that others have, pieces that are left to be done, pieces of a workgroup
};
static_assert(sizeof(State) <= kChunkLds - 2 * kStages * kPieceBytes, "it lies behind the tiles");
template <bool kE4m3>
__global__ void __launch_bounds__(kChunkThreads, 2) k_cache_chunk_even(Cache C, ChunkArgs A) {
  extern __shared__ __align__(256) char smem[];
  // XCDs get workgroups in turn, and take an eighth of all pieces each: with eight KV heads one head's, which its L2 then serves
  const int wg = (int)(blockIdx.x & 7) * (kSlots / 8) + (int)(blockIdx.x >> 3);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = (A.units + kChunkThreads - 1) / kChunkThreads, u0 = threadIdx.x * per, u1 = min(u0 + per, A.units);
  // of the units u0 .. u1 - 1 of a head, `visit` those that there are with their pieces, at least one: an empty unit is somebody's too
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
      if (W.s >= 0 && !visit(s, (int)i, max(pieces_of(C, A, W).y, 1))) return;
    }
  };
  int64_t own = 0;
  each_unit([&](int, int, int n) {
    own += n;
    return true;
  });
  int64_t upto = own;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t x = __shfl_up(upto, d);
    if (lane >= d) upto += x;
  }
  int64_t* sums = reinterpret_cast<int64_t*>(smem);
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int64_t before = upto - own, of_head = 0;
#pragma unroll
  for (int w = 0; w < kChunkWaves; ++w) {
    if (w < wave) before += sums[w];
    of_head += sums[w];
  }
  of_head = uniform(of_head);
  const int64_t total = of_head * C.hkv, share = (total + kSlots - 1) / kSlots, start = wg * share;
  if (start >= total) return;  // the whole workgroup
  int j = (int)(start / of_head);
  const int64_t at = start - j * of_head;
  if (before <= at && at < before + own) {
    int64_t sum = before;
    each_unit([&](int s, int i, int n) {
      if (at < sum + n) {
        sums[kChunkWaves] = (int64_t)s << 32 | (uint32_t)i;
        sums[kChunkWaves + 1] = at - sum;
        return false;
      }
      sum += n;
      return true;
    });
  }
  // Where the workgroup stands lies in LDS behind the tiles, and not in registers that the units want
  State* state = reinterpret_cast<State*>(smem + 2 * kStages * kPieceBytes);
  __syncthreads();
  if (threadIdx.x == 0) {
    const int64_t si = sums[kChunkWaves];
    *state = State{(int)(si >> 32), (int)si, j, 1, sums[kChunkWaves + 1], min(share, total - start), share};
  }
  __syncthreads();
  for (;;) {
    {
      const int s = __builtin_amdgcn_readfirstlane(state->s), i = __builtin_amdgcn_readfirstlane(state->i);
      const Unit W = unit_of(C, A, s, i, __builtin_amdgcn_readfirstlane(state->j));
      const int64_t q = uniform(state->q), left = uniform(state->left);
      const int n = pieces_of(C, A, W).y;
      const int64_t pieces = max(n, 1), take = min(pieces - q, left);
      const int wg = (int)(blockIdx.x & 7) * (kSlots / 8) + (int)(blockIdx.x >> 3);
      Span P;
      P.begin = (int)q;
      P.end = min((int)(q + take), n);
      P.whole = take == pieces;
      P.slot = 2 * wg + (state->first ? 0 : 1);
      if (q == 0 && threadIdx.x == 0) {
        const int64_t each = state->share;
        A.whole[(int64_t)W.j * A.units + first_unit(C, A, s) + i] = int4{P.slot, 2 * (wg + 1), P.whole ? 1 : 1 + (int)((pieces - take + each - 1) / each), 0};
      }
      __syncthreads();  // all have read the state
      if (threadIdx.x == 0) {
        state->left = left - take;
        state->q = 0;
        state->first = 0;
      }
      attend_unit<kE4m3>(C, A, W, P, smem);
    }
    __syncthreads();  // the LDS is the next unit's
    if (state->left <= 0) return;
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
    __syncthreads();  // all have read the state
    if (threadIdx.x == 0) {
      state->s = s;
      state->i = i;
      state->j = j;
    }
    __syncthreads();
  }
}

// The parts of a unit that several workgroups had: a workgroup joins 32 of its rows, a wavefront 32 channels of them.
__global__ void __launch_bounds__(256) k_cache_chunk_join(Cache C, ChunkArgs A) {
  __shared__ __align__(16) char smem[32 * kPieceRow];
  const int b = (int)(blockIdx.x >> 3), rw = (int)(blockIdx.x & 7), j = b / A.units, u = b - j * A.units;
  const int lane = threadIdx.x & 63, db = threadIdx.x >> 6, col = lane & 31, qh = lane >> 5;
  const int s = C.cu ? find_sequence(C.nseq, u, [&](int x) { return first_unit(C, A, x); }) : u;
  if (s < 0) return;
  const Unit W = unit_of(C, A, s, (int)(u - first_unit(C, A, s)), j);
  const int rows = W.nt * C.g;
  if (W.s < 0 || 32 * rw >= rows) return;
  const int4 R = A.whole[b];
  if (R.z <= 1) return;  // written already
  // (the bounds matter only if the starts of the sequences are not in order and no workgroup has written R)
  const int n = min(R.z, 2 * kSlots);
  auto slot = [&](int i) { return (int64_t)min((uint32_t)(i == 0 ? R.x : R.y + 2 * (i - 1)), 2u * kSlots - 1); };
  const int r = 32 * rw + col, rc = min(r, rows - 1), tt = div_g(rc, C.g, A.g_magic), hh = rc - tt * C.g;
  float top = -INFINITY, total = 0.f;
  f32x4 o[4];
#pragma unroll
  for (int a = 0; a < 4; ++a) o[a] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
  for (int i = 0; i < n; ++i) {
    const int64_t at = slot(i);
    const float2 x = A.part_ml[at * kChunkRows + rc];
    const f32x4* from = reinterpret_cast<const f32x4*>(A.part) + (at * kChunkWaves + rw) * 1024 + 256 * db + lane;
    f32x4 y[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) y[a] = from[64 * a];
    float f0;
    const float mc = new_reference(x.x, top, f0), f1 = __builtin_amdgcn_exp2f(x.x - mc);
    total = fmaf(total, f0, f1 * x.y);
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[a][e] = fmaf(o[a][e], f0, f1 * y[a][e]);
  }
  const bool some = total > 0.f || total != total, here = r < rows;
  const float inv = 1.f / total;
  const int64_t row = (int64_t)(W.t0 + tt) * C.hq + W.j * C.g + hh;
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
  __syncthreads();
  const int sub = threadIdx.x & 15;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int wr = 16 * i + (int)(threadIdx.x >> 4), rr = 32 * rw + wr;
    if (rr >= rows) break;
    const int t = div_g(rr, C.g, A.g_magic), h = rr - t * C.g;
    *reinterpret_cast<u32x4*>((bf16_t*)A.O + ((int64_t)(W.t0 + t) * C.hq + W.j * C.g + h) * kD + 8 * sub) =
        *reinterpret_cast<const u32x4*>(smem + wr * kPieceRow + ((sub ^ (wr & 15)) << 4));
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------------------------
struct ChunkCut {
  int tok;
  int64_t units;
  size_t ml, whole, total;  // offsets in the workspace; the sums come first
};
ChunkCut chunk_cut(const nsa_sel_cache_shape* s) {
  ChunkCut c;
  c.tok = kChunkRows / (s->hq / s->hkv);
  c.units = (int64_t)s->n_tokens / c.tok + s->nseq;
  c.ml = (size_t)2 * kSlots * kChunkRows * kD * 4;
  c.whole = c.ml + (size_t)2 * kSlots * kChunkRows * 8;
  c.total = c.whole + (size_t)c.units * s->hkv * 16;
  return c;
}
int check_chunk_shape(const nsa_sel_cache_shape* s) {
  const int rc = check_sizes(s, true);
  if (rc) return rc;
  if (s->topk != 0) return NSA_SEL_EINVAL;
  return launchable(8 * chunk_cut(s).units * s->hkv, 256) ? NSA_SEL_OK : NSA_SEL_EUNSUPPORTED;
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
  A.whole = (int4*)((char*)ws + c.whole);
  const bool e4m3 = shape->dtype == NSA_SEL_CACHE_E4M3;
  const auto kern = e4m3 ? k_cache_chunk_even<true> : k_cache_chunk_even<false>;
  static std::atomic<uint64_t> ready[2];
  if (allow_dynamic_lds((const void*)kern, kChunkLds, ready[e4m3]) != hipSuccess) return NSA_SEL_EHIP;
  {
    ProfScope ps(KID_CACHE_CHUNK, (hipStream_t)stream);
    hipLaunchKernelGGL(kern, dim3(kSlots), dim3(kChunkThreads), kChunkLds, (hipStream_t)stream, C, A);
  }
  if (hipGetLastError() != hipSuccess) return NSA_SEL_EHIP;
  ProfScope ps(KID_CACHE_CHUNK_JOIN, (hipStream_t)stream);
  hipLaunchKernelGGL(k_cache_chunk_join, dim3((unsigned)(8 * c.units * shape->hkv)), dim3(256), 0, (hipStream_t)stream, C, A);
  return hipGetLastError() == hipSuccess ? NSA_SEL_OK : NSA_SEL_EHIP;
}

}  // extern "C"
