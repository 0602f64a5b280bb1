// Attention of a few new tokens over a paged cache (nsa_sel_cache_attention): of selected blocks, of a window, or of every key.
//
// One pass over the keys with the running maximum and sum of a softmax.  What bounds it is reading the keys and values, which nothing else
// reads: 4 g flops a byte in bf16 and twice that in 8 bits, far below what the matrix cores need to be busy.  So the products may waste
// columns (of 16 a token uses g, and as many again for the rest of its probabilities), and everything serves having bytes in flight: a wavefront takes pieces of 32
// keys by itself, K straight into the registers that the product reads, V through registers into a tile of its own in LDS, and the next
// piece is requested as soon as the registers are free.  The wavefronts of a workgroup take pieces in turn and join their sums in LDS; where
// there are too few rows to fill the chip several workgroups share one, and a second kernel joins theirs.
//
// S^T = K Q^T by 16x16x32 products: a lane holds four consecutive keys of one column, and the keys of two 16-key tiles are eight
// consecutive contraction steps of O^T += V^T P^T if V's rows are read in the same order.  Nothing is transposed but V, by the LDS read.
//
// Measured: 256 tokens x 8 heads x 16 blocks of 64, bf16, 1.05 GB in 158 us, 6.6 TB/s; 8 sequences of 4096 .. 131072 tokens, g = 8, e4m3, every key,
// 0.67 GB in 111 us with the join, 6.0 TB/s; one token, 16 blocks, 6.9 us and 3.6 for the join.
//
// e4m3 values become bf16 in registers, times their page's power of two, which bf16 holds exactly: the products are those of a bf16 cache.
#include "cache.h"

namespace nsa {
namespace {

constexpr int kWaves = 4;                    // of a workgroup
constexpr int kPiece = kAttendPiece, kTiles = kPiece / 16;
constexpr int kVRow = kD * 2;                 // bytes of a row of V in LDS, its 16-byte chunks turned (row_turn)
constexpr int kSumRow = kD * 4 + 16;          // bytes of a column's sums in LDS
constexpr int kOwnLds = (16 * kSumRow + 2 * 16 * 4 + 255) & ~255;  // a wavefront's: its tile of V, and later its sums and their statistics
constexpr int kAttendLds = kWaves * kOwnLds;
static_assert(kAttendLds <= 64 * 1024, "more would have to be asked for before the first launch");
static_assert(kPiece * kVRow <= kOwnLds, "the tile of a wavefront must fit");
static_assert(64 * kWaves == kAttendThreads, "the host reckons with this many");
static_assert(kTiles == 2, "a piece is one contraction step of the PV product");

// A row of the call: `nt` consecutive new tokens t0.. of sequence s, the first of them at `place`, and KV head j.
struct Row {
  int s, t0, nt, place, j;
};
// The part of a row's pieces that a workgroup takes: [begin, end).  If that is not all of them their sums go to a place of their own, `slot`, and
// the part that begins with the first one leaves word of them for k_cache_join.
struct Part {
  int begin, end;
  bool whole;
  int slot;
  int second, count;  // slots of the row's other parts: second, second + A.slot_step, ...; with the own one `count`
};

// What a piece consists of: 16-key tiles, each in one page.
struct Piece {
  int key0;            // place of its first key
  int64_t row[kTiles];   // of the pages' rows, its first
  int rows[kTiles];      // that anything of the workgroup sees; 0 where there is no page
};
__device__ __forceinline__ float lane_float(float x, int l) {
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), l));
}

template <bool kE4m3>
struct Raw {  // a piece of K or V as it was read
  u32x4 x[kTiles * (kE4m3 ? 2 : 4)];
};

// Buffer of a tile's rows; those that nothing sees read as zero.
template <bool kE4m3>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_buffer(const char* base, const Piece& P, int i) {
  constexpr int kRow = kD * (kE4m3 ? 1 : 2);
  return buffer_of(base + P.row[i] * kRow, (uint32_t)(P.rows[i] * kRow));
}
// K: lane (row lane & 15, quarter lane >> 4) takes the 16 bytes of each contraction step that the product wants of it.
template <bool kE4m3, int kPolicy>
__device__ __forceinline__ void load_keys(const Cache& C, const Piece& P, int lane, Raw<kE4m3>& r) {
  constexpr int kRow = kD * (kE4m3 ? 1 : 2), kN = kE4m3 ? 2 : 4;
  const uint32_t off = (lane & 15) * kRow + (lane >> 4) * 16;
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    const __amdgpu_buffer_rsrc_t b = tile_buffer<kE4m3>(C.k, P, i);
#pragma unroll
    for (int s = 0; s < kN; ++s) r.x[i * kN + s] = __builtin_amdgcn_raw_buffer_load_b128(b, off + 64 * s, 0, kPolicy);
  }
}
// V: 1 KB of consecutive rows a load.
template <bool kE4m3, int kPolicy>
__device__ __forceinline__ void load_values(const Cache& C, const Piece& P, int lane, Raw<kE4m3>& r) {
  constexpr int kN = kE4m3 ? 2 : 4;
#pragma unroll
  for (int i = 0; i < kTiles; ++i) {
    const __amdgpu_buffer_rsrc_t b = tile_buffer<kE4m3>(C.v, P, i);
#pragma unroll
    for (int s = 0; s < kN; ++s) r.x[i * kN + s] = __builtin_amdgcn_raw_buffer_load_b128(b, 1024 * s + lane * 16, 0, kPolicy);
  }
}

// Row b of a call that gives every workgroup a row; s < 0 where there is none.
template <bool kGroup>
__device__ __forceinline__ Row row_of(const Cache& C, const CacheAttend& A, int b) {
  Row W;
  W.j = b % C.hkv;
  b /= C.hkv;
  if constexpr (!kGroup) {
    const TokenPlace p = token_place(C, b);
    W.s = p.s;
    W.place = p.place;
    W.t0 = b;
    W.nt = 1;
  } else {
    // groups of A.group tokens: a sequence's start at floor(cu / group) + s, room for all of them without a scan over the batch
    auto base = [&](int s) { return (int64_t)(C.cu[s] / A.group) + s; };
    W.s = find_sequence(C.nseq, b, base);
    if (W.s >= 0) {
      const int c0 = C.cu[W.s], n = C.cu[W.s + 1] - c0, i0 = (b - (int)base(W.s)) * A.group;
      W.t0 = c0 + i0;
      W.nt = min(min(A.group, n - i0), C.T - W.t0);
      W.place = C.kv_len[W.s] - n + i0;
      if (W.nt <= 0 || W.t0 < 0) W.s = -1;
    }
  }
  return W;
}

// kSelected: the pieces are those of the blocks of idx, whose column `my` of the row this lane has; else all that the row sees.  kGroup: rows of more than one token.
template <bool kE4m3, bool kSelected, bool kGroup, int kPolicy>
__device__ __forceinline__ void attend(const Cache& C, const CacheAttend& A, Row W, Part part, int my, char* smem) {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));  // what derives from it is not kept from row to row
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, qg = lane >> 4;
  // the same in every lane, and said so: the buffers below are scalar
  W.s = __builtin_amdgcn_readfirstlane(W.s);
  W.t0 = __builtin_amdgcn_readfirstlane(W.t0);
  W.nt = __builtin_amdgcn_readfirstlane(W.nt);
  W.place = __builtin_amdgcn_readfirstlane(W.place);
  W.j = __builtin_amdgcn_readfirstlane(W.j);
  part.begin = __builtin_amdgcn_readfirstlane(part.begin);
  part.end = __builtin_amdgcn_readfirstlane(part.end);
  const int limit = C.max_pages << C.page_log2;  // places that the table can name
  // this lane's column: token tt of the group, head hh; it sees the places [c_lo, c_hi).  Without groups column c + 8 is c's again.
  const int own_col = kGroup ? col : col & 7, tt = kGroup ? col / C.g : 0, hh = own_col - tt * C.g, cols = W.nt * C.g;
  const bool used = own_col < cols;
  // what any column sees, and what all of them see
  const int lo = A.window > 0 ? max(W.place + 1 - A.window, 0) : 0, hi = min(W.place + W.nt, limit);
  const int all_lo = A.window > 0 ? max(W.place + W.nt - A.window, 0) : 0, all_hi = min(W.place + 1, limit);
  // (what the unused columns see does not matter)
  const int c_hi = kGroup ? min(W.place + tt + 1, limit) : hi, c_lo = kGroup && A.window > 0 ? max(W.place + tt + 1 - A.window, 0) : lo;

  bf16x8 qf[4];
  {
    const bf16_t* src = (const bf16_t*)A.Q + ((int64_t)(W.t0 + (used ? tt : 0)) * C.hq + W.j * C.g + (used ? hh : 0)) * kD;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      // e4m3: the 16 bytes a lane reads are two contraction steps
      const int d = kE4m3 ? 64 * (s >> 1) + 16 * qg + 8 * (s & 1) : 32 * s + 8 * qg;
      u32x4 x = *reinterpret_cast<const u32x4*>(src + d);
      if (!used) x = u32x4{0u, 0u, 0u, 0u};
      qf[s] = __builtin_bit_cast(bf16x8, x);
    }
  }

  // the pieces: of the kept blocks in their order, or all from lo to hi
  int n_pieces, first_piece = 0, blocks = 0;
  const int per_block = A.block / kPiece;
  if constexpr (kSelected) {
    const int64_t b0 = (int64_t)my * A.block;
    const bool ok = my >= 0 && b0 < hi && b0 + A.block > lo;
    const uint64_t okm = __builtin_amdgcn_ballot_w64(ok);
    uint64_t keep = 0;
    for (int m = 0; m < A.topk; ++m) {
      if (!((okm >> m) & 1)) continue;
      const int x = __builtin_amdgcn_readlane(my, m);
      const uint64_t same = __builtin_amdgcn_ballot_w64(ok && my == x) & ((1ull << m) - 1ull);
      if (same == 0) keep |= 1ull << m;
    }
    // lane i gets the i-th kept block
    const int below = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(keep >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)keep, 0));
    const int to = ((keep >> lane) & 1) ? below : 63 - (lane - below);
    blocks = __builtin_amdgcn_ds_permute(to << 2, my);
    n_pieces = __builtin_popcountll(keep) * per_block;
  } else {
    first_piece = lo / kPiece;
    n_pieces = max((hi + kPiece - 1) / kPiece - first_piece, 0);
  }

  // this workgroup's pieces, its wavefronts in turn; their places, pages and scales are looked up kAhead at a time, piece lane / kTiles of
  // these and its tile lane % kTiles
  constexpr int kAhead = 64 / kTiles;
  if constexpr (kSelected) {  // how many parts there are is known only now
    const int n = max((n_pieces + A.chunk - 1) / A.chunk, 1);
    if (part.begin >= n * A.chunk) return;  // the whole workgroup
    part.whole = n == 1;
    part.count = n;
  }
  const int begin = part.begin, end = min(part.end, n_pieces);
  const int w0 = begin + wave;
  const int mine = end > w0 ? (end - w0 + kWaves - 1) / kWaves : 0;
  int key_of = 0, rows_of = 0;
  int64_t row_of = 0;
  float k_scale = 1.f, v_scale = 1.f;
  auto look_up = [&](int i) __attribute__((always_inline)) {
    const int p = w0 + (i + lane / kTiles) * kWaves, pc = min(p, end - 1);
    if constexpr (kSelected) {
      const int o = pc / per_block;
      const int id = (int)lane_value((uint32_t)blocks, o);
      key_of = id * A.block + (pc - o * per_block) * kPiece;
    } else {
      key_of = (first_piece + pc) * kPiece;
    }
    const int key = key_of + 16 * (lane % kTiles), page = p < end ? page_of(C, W.s, key) : -1;
    rows_of = page < 0 ? 0 : min(max(hi - key, 0), 16);
    const int64_t at = (int64_t)max(page, 0) * C.hkv + W.j;
    row_of = (at << C.page_log2) + (key & ((1 << C.page_log2) - 1));
    if constexpr (kE4m3) {
      if (page >= 0) {
        k_scale = C.ks[at];
        v_scale = C.vs[at];
      }
    }
  };
  auto piece = [&](int i) __attribute__((always_inline)) {
    Piece P;
    const int l = (i % kAhead) * kTiles;
    P.key0 = __builtin_amdgcn_readlane(key_of, l);
#pragma unroll
    for (int x = 0; x < kTiles; ++x) {
      P.rows[x] = __builtin_amdgcn_readlane(rows_of, l + x);
      P.row[x] = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(row_of >> 32), l + x) << 32 |
                           (uint32_t)__builtin_amdgcn_readlane((int)row_of, l + x));
    }
    return P;
  };

  const float c2 = A.scale * 1.4426950408889634f;
  float m_run = -INFINITY, l_run = 0.f;
  f32x4 oacc[8];
#pragma unroll
  for (int d = 0; d < 8; ++d) oacc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  const uint32_t v_lds = lds_address(smem) + wave * kOwnLds;
  // V^T operand of channels 16 d ..: rows (col / 4) + 4 qg and those 16 on, columns 16 d + 4 (col % 4).  The tile lies at a multiple of 256
  // bytes, so a chunk's place is flipped into the address; done anew for every piece, it takes no registers.
  const int v_row = (col >> 2) + 4 * qg;
  const uint32_t v_at = v_lds + v_row * kVRow + ((((col & 3) >> 1) ^ row_turn(v_row)) << 4) + 8 * (col & 1);
  auto values = [&](uint32_t at, int d) __attribute__((always_inline)) {
    const uint32_t a = at ^ (d << 5);
    return __builtin_shufflevector(lds_read_tr_at(a), lds_read_tr_at(a + 16 * kVRow), 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // where this lane's 16 bytes of a load go (e4m3: the first of two chunks): row lane / 16 of four (lane / 8 of eight), whose turn the
  // later rows of the tile flip further
  const int w_row = kE4m3 ? lane >> 3 : lane >> 4;
  const uint32_t w_at = v_lds + w_row * kVRow + (((kE4m3 ? 2 * (lane & 7) : col) ^ row_turn(w_row)) << 4);
  Raw<kE4m3> kr, vr;
  Piece P;
  if (mine > 0) {
    look_up(0);
    P = piece(0);
    load_keys<kE4m3, kPolicy>(C, P, lane, kr);
    load_values<kE4m3, kPolicy>(C, P, lane, vr);
  }
  for (int i = 0; i < mine; ++i) {
    const Piece cur = P;
    float ks[kTiles], vs[kTiles];  // (taken here and not with the piece: its loads need not wait for those of the scales)
#pragma unroll
    for (int x = 0; x < kTiles; ++x) {
      ks[x] = kE4m3 ? lane_float(k_scale, (i % kAhead) * kTiles + x) : 1.f;
      vs[x] = kE4m3 ? lane_float(v_scale, (i % kAhead) * kTiles + x) : 1.f;
    }
    f32x4 sacc[kTiles];
#pragma unroll
    for (int x = 0; x < kTiles; ++x) {
      sacc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        u32x4 a;
        if constexpr (kE4m3) {
          const u32x4 r = kr.x[2 * x + (s >> 1)];
          a = (s & 1) ? eight_bf16(r[2], r[3], ks[x]) : eight_bf16(r[0], r[1], ks[x]);
        } else {
          a = kr.x[4 * x + s];
        }
        sacc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), qf[s], sacc[x], 0, 0, 0);
      }
    }
    const bool more = i + 1 < mine;
    if (more) {
      if ((i + 1) % kAhead == 0) look_up(i + 1);
      P = piece(i + 1);
      load_keys<kE4m3, kPolicy>(C, P, lane, kr);
    }
    // scores of places that the column does not see become -inf
    bool whole = cur.key0 >= all_lo && cur.key0 + kPiece <= all_hi;
#pragma unroll
    for (int x = 0; x < kTiles; ++x) whole = whole && cur.rows[x] > 0;
    float m = -INFINITY;
    if (!whole) {
#pragma unroll
      for (int x = 0; x < kTiles; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = cur.key0 + 16 * x + 4 * qg + e;
          if (key < c_lo || key >= c_hi || cur.rows[x] == 0) sacc[x][e] = -INFINITY;
        }
    }
#pragma unroll
    for (int x = 0; x < kTiles; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) m = fmaxf(m, sacc[x][e]);
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    const float m_new = fmaxf(m_run, m);
    const float mc = m_new == -INFINITY ? 0.f : m_new * c2;
    const float alpha = __builtin_amdgcn_exp2f(fmaf(m_run, c2, -mc));  // exp2(-inf) = 0 on the first piece with a score
    m_run = m_new;
    // A probability goes into the product in two parts, the bf16 value below it and the rest as bf16, so that its first 16 bits count: as one bf16
    // value it would lose up to 2^-8 of itself, and sums of values that cancel up to five times what the rounding of O does.  The rest is zero only where the
    // probability is: zero times an infinite value would be NaN.  Without groups the columns from 8 on, which repeat the others, have it; a group's may all be in use, and
    // it is a product of its own.
    float l = 0.f;
    bf16x8 pf, pr;
#pragma unroll
    for (int x = 0; x < kTiles; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __builtin_amdgcn_exp2f(fmaf(sacc[x][e], c2, -mc));
        l += p;
        const float high = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, p) & 0xffff0000u), rest = fmaxf(p - high, fminf(p, 0x1p-126f));
        pf[4 * x + e] = (bf16_t)(kGroup || col < 8 ? high : rest);
        if constexpr (kGroup) pr[4 * x + e] = (bf16_t)rest;
      }
    l_run = fmaf(l_run, alpha, l);
#pragma unroll
    for (int d = 0; d < 8; ++d) oacc[d] *= alpha;
    uint32_t va = v_at, wa = w_at;
    asm volatile("" : "+v"(va), "+v"(wa));  // what derives from them is not kept from piece to piece
    // V into this wavefront's tile; rows before anything that the group sees as zeros, whatever they hold
#pragma unroll
    for (int x = 0; x < kTiles; ++x) {
      constexpr int kN = kE4m3 ? 2 : 4;
#pragma unroll
      for (int s = 0; s < kN; ++s) {
        u32x4 r = vr.x[x * kN + s];
        const int row = 16 * x + (kE4m3 ? 8 : 4) * s;
        if (cur.key0 + row + w_row < lo) r = u32x4{0u, 0u, 0u, 0u};
        const uint32_t at = (wa ^ (row_turn(row) << 4)) + row * kVRow;
        if constexpr (kE4m3) {
          lds_write_16(at, eight_bf16(r[0], r[1], vs[x]));
          lds_write_16(at ^ 16, eight_bf16(r[2], r[3], vs[x]));
        } else {
          lds_write_16(at, r);
        }
      }
    }
    if (more) load_values<kE4m3, kPolicy>(C, P, lane, vr);
    wave_sync();
    if (!kGroup || (cur.key0 >= all_lo && cur.key0 + kPiece <= all_hi)) {
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        const bf16x8 a = values(va, d);
        oacc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pf, oacc[d], 0, 0, 0);
        if constexpr (kGroup) oacc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pr, oacc[d], 0, 0, 0);
      }
    } else {
      // Tokens of the group see different keys of the piece, and what one does not see may be an infinity or a NaN, which a
      // probability of zero does not silence: one token at a time, the others' keys as zeros.
      for (int k = 0; k < W.nt; ++k) {
        const int k_hi = min(W.place + k + 1, limit) - cur.key0, k_lo = (A.window > 0 ? max(W.place + k + 1 - A.window, 0) : 0) - cur.key0;
#pragma unroll
        for (int d = 0; d < 8; ++d) {
          bf16x8 a = values(va, d);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int key = 16 * (e >> 2) + 4 * qg + (e & 3);
            if (key < k_lo || key >= k_hi) a[e] = (bf16_t)0.f;
          }
          f32x4 add = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pf, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
          add = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pr, add, 0, 0, 0);
          if (tt == k) oacc[d] += add;
        }
      }
    }
    wave_sync();  // the tile is overwritten by the next piece
  }
  l_run += __shfl_xor(l_run, 16);
  l_run += __shfl_xor(l_run, 32);

  // join the four wavefronts
  {
    char* own = smem + wave * kOwnLds;
#pragma unroll
    for (int d = 0; d < 8; ++d) *reinterpret_cast<f32x4*>(own + col * kSumRow + (16 * d + 4 * qg) * 4) = oacc[d];
    if (qg == 0) {
      reinterpret_cast<float*>(own + 16 * kSumRow)[col] = m_run;
      reinterpret_cast<float*>(own + 16 * kSumRow)[16 + col] = l_run;
    }
  }
  __syncthreads();
  const int c = tid >> 4, sub = tid & 15;
  if (part.begin == 0 && A.rows != nullptr && c < W.nt && sub == 0)
    A.rows[(int64_t)(W.t0 + c) * C.hkv + W.j] = int4{part.slot, part.second, part.whole ? 1 : part.count, W.t0};
  if (c >= cols) return;
  float top = -INFINITY, total = 0.f, o[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) top = fmaxf(top, reinterpret_cast<const float*>(smem + w * kOwnLds + 16 * kSumRow)[c]);
  const float tc = top == -INFINITY ? 0.f : top * c2;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const char* from = smem + w * kOwnLds;
    const float* ml = reinterpret_cast<const float*>(from + 16 * kSumRow);
    const float f = __builtin_amdgcn_exp2f(fmaf(ml[c], c2, -tc));
    total = fmaf(f, ml[16 + c], total);
    f32x4 a = *reinterpret_cast<const f32x4*>(from + c * kSumRow + 32 * sub), b = *reinterpret_cast<const f32x4*>(from + c * kSumRow + 32 * sub + 16);
    if constexpr (!kGroup) {
      a += *reinterpret_cast<const f32x4*>(from + (c + 8) * kSumRow + 32 * sub);
      b += *reinterpret_cast<const f32x4*>(from + (c + 8) * kSumRow + 32 * sub + 16);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[e] = fmaf(f, a[e], o[e]);
      o[4 + e] = fmaf(f, b[e], o[4 + e]);
    }
  }
  const int ct = kGroup ? c / C.g : 0;
  const int64_t row = (int64_t)(W.t0 + ct) * C.hq + W.j * C.g + (c - ct * C.g);
  if (!part.whole) {
    const int64_t at = (int64_t)part.slot * A.cols + c;
    float* dst = A.part + at * kD + 8 * sub;
    *reinterpret_cast<f32x4*>(dst) = f32x4{o[0], o[1], o[2], o[3]};
    *reinterpret_cast<f32x4*>(dst + 4) = f32x4{o[4], o[5], o[6], o[7]};
    if (sub == 0) A.part_ml[at] = float2{top, total};
    return;
  }
  const bool some = total > 0.f || total != total;
  const float inv = 1.f / total;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = some ? o[e] * inv : 0.f;  // an empty row is 0 whatever its values are
  if (A.gate) {
    const float gate = A.gate[row];
    u32x4 x = u32x4{0u, 0u, 0u, 0u};
    if (A.o_acc) x = *reinterpret_cast<const u32x4*>((const bf16_t*)A.o_acc + row * kD + 8 * sub);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[2 * e] = fmaf(gate, o[2 * e], bf16_lo(x[e]));
      o[2 * e + 1] = fmaf(gate, o[2 * e + 1], bf16_hi(x[e]));
    }
  }
  u32x4 x;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = pack_bf16x2(o[2 * e], o[2 * e + 1]);
  *reinterpret_cast<u32x4*>((bf16_t*)A.O + row * kD + 8 * sub) = x;
  if (sub == 0) A.LSE[row] = some ? (tc + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
}

// A row a workgroup, or with A.splits the `chunk` pieces of a row that are its own.
template <bool kE4m3, bool kSelected, bool kGroup, int kPolicy>
__global__ void __launch_bounds__(64 * kWaves, kGroup ? 2 : 3) k_cache_attend(Cache C, CacheAttend A) {
  extern __shared__ __align__(256) char smem[];
  // all rows' first parts before the second ones: those that a short row leaves empty come last, and the XCDs, which get workgroups in
  // turn, have as much to do each
  const int rows = (int)gridDim.x / A.splits, split = (int)blockIdx.x / rows, b = (int)blockIdx.x - split * rows;
  // this lane's column of idx, requested before the sequence and its length are known
  const int lane = threadIdx.x & 63, my = kSelected && lane < A.topk ? A.idx[(int64_t)b * A.topk + lane] : -1;
  const Row W = row_of<kGroup>(C, A, b);
  if (W.s < 0) return;  // the whole workgroup
  Part P;
  P.begin = split * A.chunk;
  P.end = P.begin + A.chunk;
  P.whole = true;
  P.slot = b * A.splits + split;
  P.second = P.slot + 1;
  P.count = 1;
  attend<kE4m3, kSelected, kGroup, kPolicy>(C, A, W, P, my, smem);
}

// Every key of sequences whose lengths only the device knows: all pieces of all rows, one row after the other, are cut into 512 equal parts, so
// that all workgroups end together whatever the lengths.  A workgroup finds its sequence by a scan over the batch's lengths.  Its part may begin
// and end inside a row; rows in between are its own.  Measured against parts of 1024 keys, with room for the longest row everywhere, joined by
// row: 8 sequences of 4096 .. 131072, e4m3, 64 heads, g = 8, 139 -> 120 us; one of 65536, bf16, 32 heads 57 -> 54; 64 of 100 .. 32000 286 -> 267.  More
// parts than 512 (768, 1024, 1536) cost up to 6 % but in the last case (256 us for 1536).
__device__ __forceinline__ int64_t uniform(int64_t x) {  // a value that all lanes have, in scalar registers
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
}
template <bool kE4m3, bool kGroup, int kPolicy>
__global__ void __launch_bounds__(64 * kWaves, kGroup ? 2 : 3) k_cache_attend_even(Cache C, CacheAttend A) {
  extern __shared__ __align__(256) char smem[];
  const int limit = C.max_pages << C.page_log2, n_wg = (int)gridDim.x, wg = (int)blockIdx.x;
  auto pieces_of = [&](int s) __attribute__((always_inline)) {  // of each row of sequence s, no fewer than any of them has
    const int n = (min(C.kv_len[s], limit) + kPiece - 1) / kPiece;
    return max(A.window > 0 ? min(n, (A.window + A.group) / kPiece + 2) : n, 1);
  };
  auto groups_of = [&](int s) __attribute__((always_inline)) { return C.cu ? (max(C.cu[s + 1] - C.cu[s], 0) + A.group - 1) / A.group : 1; };
  // exclusive sums over the batch: a run of `per` sequences a thread
  const int per = (C.nseq + 64 * kWaves - 1) / (64 * kWaves), s0 = threadIdx.x * per, lane = threadIdx.x & 63;
  int64_t own = 0;
  for (int s = s0; s < min(s0 + per, C.nseq); ++s) own += (int64_t)groups_of(s) * C.hkv * pieces_of(s);
  int64_t upto = own;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t x = __shfl_up(upto, d);
    if (lane >= d) upto += x;
  }
  int64_t* sums = reinterpret_cast<int64_t*>(smem);
  if (lane == 63) sums[threadIdx.x >> 6] = upto;
  __syncthreads();
  int64_t before = upto - own, total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < (int)(threadIdx.x >> 6)) before += sums[w];
    total += sums[w];
  }
  total = uniform(total);
  const int64_t share = max((total + n_wg - 1) / n_wg, (int64_t)kWaves), start = wg * share;
  if (start >= total) return;  // the whole workgroup
  if (before <= start && start < before + own) {
    sums[kWaves] = s0;
    sums[kWaves + 1] = before;
  }
  __syncthreads();
  int s = __builtin_amdgcn_readfirstlane((int)sums[kWaves]);
  int64_t at = start - uniform(sums[kWaves + 1]);
  __syncthreads();
  int groups = groups_of(s), pieces = pieces_of(s);
  while (at >= (int64_t)groups * C.hkv * pieces) {
    at -= (int64_t)groups * C.hkv * pieces;
    ++s;
    groups = groups_of(s);
    pieces = pieces_of(s);
  }
  int unit = __builtin_amdgcn_readfirstlane((int)(at / pieces)), q = __builtin_amdgcn_readfirstlane((int)(at - (int64_t)unit * pieces));
  const int each = __builtin_amdgcn_readfirstlane((int)share);  // below 2^31: checked on the host
  int left = __builtin_amdgcn_readfirstlane((int)min(share, total - start));
  for (bool first = true; left > 0; first = false) {
    const int take = min(pieces - q, left), i = unit / C.hkv;
    Row W;
    W.s = s;
    W.j = unit - i * C.hkv;
    const int c0 = C.cu ? C.cu[s] : s, n = C.cu ? C.cu[s + 1] - c0 : 1, i0 = i * A.group;
    W.t0 = c0 + i0;
    W.nt = min(min(A.group, n - i0), C.T - W.t0);
    W.place = C.kv_len[s] - n + i0;
    Part P;
    P.begin = q;
    P.end = q + take;
    P.whole = take == pieces;
    P.slot = 2 * wg + (first ? 0 : 1);
    P.second = 2 * (wg + 1);
    P.count = 1 + (pieces - take + each - 1) / each;
    if (W.nt > 0 && W.t0 >= 0) attend<kE4m3, false, kGroup, kPolicy>(C, A, W, P, -1, smem);
    left -= take;
    q = 0;
    if (++unit == groups * C.hkv && left > 0) {
      unit = 0;
      do {
        ++s;
        groups = groups_of(s);
      } while (groups == 0);
      pieces = pieces_of(s);
    }
    __syncthreads();  // the LDS is the next row's
  }
}

// The parts of a row: a workgroup a row, whose groups of 16 lanes, 8 channels a lane, take them in turn.
__global__ void __launch_bounds__(kJoinThreads) k_cache_join(Cache C, CacheAttend A) {
  __shared__ float sums[16][kD + 4], stats[16];
  const int64_t row = blockIdx.x;
  const int t = (int)(row / C.hq), h = (int)(row - (int64_t)t * C.hq), grp = threadIdx.x >> 4, sub = threadIdx.x & 15;
  if (C.cu && (t < C.cu[0] || t >= C.cu[C.nseq])) return;  // rows of no sequence are left as they were
  const int4 R = A.rows[(int64_t)t * C.hkv + h / C.g];
  if (R.z <= 1) return;  // written already
  // (the bounds matter only if the starts of the sequences are not in order and no workgroup has written R)
  const int n = min(R.z, A.slots), col = min(max(t - R.w, 0) * C.g + h % C.g, A.cols - 1);
  auto slot = [&](int i) { return (int64_t)min((uint32_t)(i == 0 ? R.x : R.y + (i - 1) * A.slot_step), (uint32_t)A.slots - 1) * A.cols + col; };
  const float c2 = A.scale * 1.4426950408889634f;
  float top = -INFINITY;
  for (int i = sub; i < n; i += 16) top = fmaxf(top, A.part_ml[slot(i)].x);
#pragma unroll
  for (int m = 1; m < 16; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
  const float tc = top == -INFINITY ? 0.f : top * c2;
  float total = 0.f, o[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = 0.f;
#pragma unroll 2
  for (int i = grp; i < n; i += 16) {
    const int64_t at = slot(i);
    const float2 x = A.part_ml[at];
    const float* from = A.part + at * kD + 8 * sub;
    const f32x4 a = *reinterpret_cast<const f32x4*>(from), b = *reinterpret_cast<const f32x4*>(from + 4);
    const float f = __builtin_amdgcn_exp2f(fmaf(x.x, c2, -tc));
    total = fmaf(f, x.y, total);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[e] = fmaf(f, a[e], o[e]);
      o[4 + e] = fmaf(f, b[e], o[4 + e]);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[grp][8 * sub + e] = o[e];
  if (sub == 0) stats[grp] = total;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  const int lane = threadIdx.x;
  float p = 0.f, q = 0.f;
  total = 0.f;
#pragma unroll
  for (int g = 0; g < 16; ++g) {
    p += sums[g][2 * lane];
    q += sums[g][2 * lane + 1];
    total += stats[g];
  }
  const bool some = total > 0.f || total != total;
  const float inv = 1.f / total;
  p = some ? p * inv : 0.f;
  q = some ? q * inv : 0.f;
  if (A.gate) {
    const float gate = A.gate[row];
    const uint32_t x = A.o_acc ? reinterpret_cast<const uint32_t*>(A.o_acc)[row * (kD / 2) + lane] : 0u;
    p = fmaf(gate, p, bf16_lo(x));
    q = fmaf(gate, q, bf16_hi(x));
  }
  reinterpret_cast<uint32_t*>(A.O)[row * (kD / 2) + lane] = pack_bf16x2(p, q);
  if (lane == 0) A.LSE[row] = some ? (tc + __builtin_amdgcn_logf(total)) * 0.6931471805599453f : -INFINITY;
}

}  // namespace

hipError_t launch_cache_attend(const Cache& C, bool e4m3, const CacheAttend& A, hipStream_t st) {
  const bool grouped = A.group > 1;
  using Kernel = void (*)(Cache, CacheAttend);
#define FORMS(e4m3, policy)                                                                                           \
  k_cache_attend<e4m3, true, false, policy>, k_cache_attend<e4m3, false, false, policy>,                              \
      k_cache_attend_even<e4m3, false, policy>
  static const Kernel kForms[16] = {FORMS(false, 0), k_cache_attend<false, false, true, 0>, FORMS(false, kNonTemporal), k_cache_attend_even<false, true, 0>,
                                    FORMS(true, 0),  k_cache_attend<true, false, true, 0>,  FORMS(true, kNonTemporal),  k_cache_attend_even<true, true, 0>};
#undef FORMS
  const int form = (e4m3 ? 8 : 0) + (grouped ? (A.even > 0 ? 7 : 3) : (A.streaming ? 4 : 0) + (A.idx ? 0 : A.even > 0 ? 2 : 1));
  const Kernel kern = kForms[form];
  {
    ProfScope ps(KID_CACHE_ATTEND, st);
    hipLaunchKernelGGL(kern, dim3((unsigned)A.workgroups), dim3(kAttendThreads), kAttendLds, st, C, A);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || A.rows == nullptr) return e;
  ProfScope ps(KID_CACHE_JOIN, st);
  hipLaunchKernelGGL(k_cache_join, dim3((unsigned)((int64_t)C.T * C.hq)), dim3(kJoinThreads), 0, st, C, A);
  return hipGetLastError();
}

}  // namespace nsa
