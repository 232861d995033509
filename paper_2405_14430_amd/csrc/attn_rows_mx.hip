// Attention of packed rows over pages of 8- or 4-bit numbers: the kernels of attn_rows.h with a loader that brings codes from memory and
// writes what they stand for to LDS, in the type of the rows.
//
// Every value that the pages can hold is a number of both types, so from the LDS on nothing differs from pages of rows, and the tile, key and
// wide kernels' results are bit for bit those over pages that hold the decoded rows.  A tile needs half or a quarter of the bytes from memory, and a
// conversion instruction for two channels on its way to LDS.  The few kernel below has tiles, chunks and an order of sums of its own: its results are the
// same but for rounding.
#include "attn_rows.h"
#include "mx.h"

namespace pf {
namespace {

// The interface of TileLoader.  A lane's share of a load is a unit of UNIT neighbouring channels of a row (up to 16 bytes of codes) and
// their block's exponent; it goes to LDS in pieces of 16 bytes, as many in all as TileLoader has loads.
template <typename C, typename T, int SRC>
struct MxTileLoader : PageWalk<C::TK> {
  static constexpr int FMT = SRC == KEYS_E4M3 ? PF_MX_E4M3 : PF_MX_E2M1, BITS = Mx<FMT>::BITS;
  static constexpr int TK = C::TK, DHP = C::ROWB / (int)sizeof(T);
  static constexpr int GROWS = C::RW > 16 ? 16 : C::RW, GROUPS = C::RW / GROWS;   // a load's rows lie in one group of 16 keys
  // the largest unit with which whole loads of 64 lanes make up a group's rows
  static constexpr int unit() {
    for (int u = 128 / BITS; u > 2; u /= 2)
      if (GROWS * DHP % (64 * u) == 0) return u;
    return 0;
  }
  static constexpr int UNIT = unit(), BYTES = UNIT * BITS / 8, WORDS = BYTES < 4 ? 1 : BYTES / 4;
  static constexpr int UPR = DHP / UNIT;                           // units to a row
  static constexpr int GL = GROWS * UPR / 64, LOADS = GROUPS * GL; // loads per group, and per tile
  static constexpr int PIECE = 16 / (int)sizeof(T), PIECES = UNIT / PIECE;
  static_assert(UNIT >= PIECE && UNIT <= PF_MX_BLOCK && LOADS * PIECES == C::LOADS, "a unit is whole pieces of one block");
  static constexpr unsigned kOutside = 0x7fff0000u;
  const RowsAttn &a;
  const int lane, lw, s, kb, ke;
  // The lane's bytes from a group's first row, where its exponent is, and where the unit goes in an LDS tile.  Where a load is a whole
  // number of rows its lanes' places are those of the first one, so many rows further.
  static constexpr bool WHOLE = 64 % UPR == 0;
  static constexpr int OFFS = WHOLE ? 1 : GL, RPL = 64 / UPR;
  unsigned off[OFFS], scale_off[OFFS];
  int k_lds[OFFS], v_lds[OFFS];
  const uint8_t *k_head, *v_head, *ks_head, *vs_head;
  const uint8_t *k_from[GROUPS], *v_from[GROUPS], *ks_from[GROUPS], *vs_from[GROUPS];
  int in_group[GROUPS];                                            // rows of the group that there are
  unsigned k_reg[LOADS][WORDS], v_reg[LOADS][WORDS], k_exp[LOADS][1], v_exp[LOADS][1];

  __device__ __forceinline__ MxTileLoader(const RowsAttn &args, const Work &w, int lane_, int lw_, int kb_, int ke_)
      : a(args), lane(lane_), lw(lw_), s(w.s), kb(kb_), ke(ke_) {
#pragma unroll
    for (int i = 0; i < OFFS; ++i) {
      const int u = i * 64 + lane, row = u / UPR, c = u % UPR * UNIT, byte = c * BITS / 8;
      const bool there = byte < a.mx.row_bytes;                    // rows of codes are whole units of 16 bytes
      unsigned at = row * a.mx.row_bytes + byte, scale_at = row * a.mx.blocks + c / PF_MX_BLOCK;
      asm volatile("" : "+v"(at), "+v"(scale_at));                 // selected, not branched around: the build looks at moves in branches
      off[i] = there ? at : kOutside;
      scale_off[i] = there ? scale_at : kOutside;
      k_lds[i] = (lw * C::RW + row) * C::KROWB + c * (int)sizeof(T);
      v_lds[i] = (lw * C::RW + row) * C::VROWB + c * (int)sizeof(T);
    }
    const int64_t row0 = (int64_t)w.hk << a.pages.page_shift;
    k_head = (const uint8_t *)a.pages.k + row0 * a.mx.row_bytes;
    v_head = (const uint8_t *)a.pages.v + row0 * a.mx.row_bytes;
    ks_head = a.mx.k_scale + row0 * a.mx.blocks;
    vs_head = a.mx.v_scale + row0 * a.mx.blocks;
    this->start(a, lane, s, kb, ke);
  }
  // Sets the sources of tile t's loads.  Tiles have to be taken in order, each once; tiles behind the last one read as zeros.
  __device__ __forceinline__ void aim(int t) {
    this->take(a, lane, s, kb, ke, t);
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int key = kb + t * TK + lw * C::RW + g * GROWS;        // wave-uniform
      const int pg = this->of(t, lw * C::RW + g * GROWS);
      const int row = key & ((1 << a.pages.page_shift) - 1);
      const int64_t page = pg < 0 ? 0 : pg;
      k_from[g] = uniform(k_head + page * a.pages.k_stride + row * a.mx.row_bytes);
      v_from[g] = uniform(v_head + page * a.pages.v_stride + row * a.mx.row_bytes);
      ks_from[g] = uniform(ks_head + page * a.mx.k_scale_stride + row * a.mx.blocks);
      vs_from[g] = uniform(vs_head + page * a.mx.v_scale_stride + row * a.mx.blocks);
      in_group[g] = uniform(pg < 0 ? 0 : clampi(ke - key, 0, GROWS));
    }
  }
  // TileLoader's: in tiles with keys that some row does not see, values that are infinities or NaN are taken out of the registers and
  // noted.  append writes none but NaN of whole blocks, but a page that nothing was written to may hold anything.  A code is not finite from
  // a magnitude `least` on: e4m3 7f, and where the block's power is too large the codes that reach 2^128 with it; byte 255: all.  The
  // codes of a word are compared together, in the bits of their signs.
  __device__ __forceinline__ void clear_v(unsigned *hidden, int at) {
    constexpr unsigned kOnes = BITS == 8 ? 0x01010101u : 0x11111111u, kSigns = kOnes << (BITS - 1);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const unsigned byte = v_exp[i][0];
      const unsigned least = byte == 255 ? 0 : BITS == 8 ? min(127u, (262 - byte) * 8) : min(8u, (256 - byte) * 2);
      unsigned bad = 0;
#pragma unroll
      for (int e = 0; e < WORDS; ++e) {
        const unsigned over = ((v_reg[i][e] & ~kSigns) + ((1u << (BITS - 1)) - least) * kOnes) & kSigns;
        const unsigned mask = (over << 1) - (over >> (BITS - 1));
        v_reg[i][e] &= ~mask;
        bad |= mask;
      }
      v_exp[i][0] = byte == 255 ? 0 : byte;                        // nothing is left of a block of NaN
      const int row = lw * C::RW + i / GL * GROWS + (i % GL * 64 + lane) / UPR;
      if (bad) atomicOr(hidden + at * (TK / 32) + (row >> 5), 1u << (row & 31));
    }
  }
  // One row of the values, for a key that there is.
  struct ValueRow {
    bool there;
    const uint8_t *code, *exp;
    __device__ __forceinline__ ValueRow(const RowsAttn &a, const Work &w, int key) {
      const int pg = a.pages.table[(int64_t)w.s * a.pages.max_pages + (key >> a.pages.page_shift)];
      there = pg >= 0 && pg < a.pages.n_pages;
      const int64_t row = ((int64_t)w.hk << a.pages.page_shift) + (key & ((1 << a.pages.page_shift) - 1));
      code = (const uint8_t *)a.pages.v + pg * a.pages.v_stride + row * a.mx.row_bytes;
      exp = a.mx.v_scale + pg * a.mx.v_scale_stride + row * a.mx.blocks;
    }
    __device__ __forceinline__ float operator[](int c) const {
      const unsigned byte = code[c * BITS / 8];
      return mx_decode_f32<FMT, 0>(BITS == 4 && (c & 1) ? byte >> 4 : byte, mx_power(exp[c / PF_MX_BLOCK])).x;
    }
  };
  __device__ __forceinline__ void get(int i, const uint8_t *from, const uint8_t *scale_from, unsigned (&reg)[WORDS], unsigned (&exp)[1]) {
    const int l = i % GL, o = WHOLE ? 0 : l, rows = WHOLE ? l * RPL : 0;
    Buffer<C::POLICY>(from, in_group[i / GL] * a.mx.row_bytes).template load<BYTES>(reg, off[o], rows * a.mx.row_bytes);
    Buffer<C::POLICY>(scale_from, in_group[i / GL] * a.mx.blocks).template load<1>(exp, scale_off[o], rows * a.mx.blocks);
  }
  // Step i of C::LOADS of a tile: a load is made when the last piece of its registers has gone to LDS.
  __device__ __forceinline__ void load_k(int i) {
    if (i % PIECES == PIECES - 1) get(i / PIECES, k_from[i / PIECES / GL], ks_from[i / PIECES / GL], k_reg[i / PIECES], k_exp[i / PIECES]);
  }
  __device__ __forceinline__ void load_v(int i) {
    if (i % PIECES == PIECES - 1) get(i / PIECES, v_from[i / PIECES / GL], vs_from[i / PIECES / GL], v_reg[i / PIECES], v_exp[i / PIECES]);
  }
  __device__ __forceinline__ void load(int t) {
    aim(t);
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) load_k(i);
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) load_v(i);
  }
  // Piece p of a unit: PIECE channels from channel p * PIECE on, decoded.
  __device__ __forceinline__ static u32x4 piece(const unsigned (&reg)[WORDS], unsigned exp, int p) {
    const float power = mx_power(exp);
    u32x4 x;
    if constexpr (sizeof(T) == 2 && FMT == PF_MX_E4M3) {
      x = u32x4{mx_decode_bf16<FMT, 0>(reg[2 * p], power), mx_decode_bf16<FMT, 1>(reg[2 * p], power),
                mx_decode_bf16<FMT, 0>(reg[2 * p + 1], power), mx_decode_bf16<FMT, 1>(reg[2 * p + 1], power)};
    } else if constexpr (sizeof(T) == 2) {
      x = u32x4{mx_decode_bf16<FMT, 0>(reg[p], power), mx_decode_bf16<FMT, 1>(reg[p], power), mx_decode_bf16<FMT, 2>(reg[p], power),
                mx_decode_bf16<FMT, 3>(reg[p], power)};
    } else {
      float2 lo, hi;
      if constexpr (FMT == PF_MX_E4M3) {
        lo = mx_decode_f32<FMT, 0>(reg[p], power);
        hi = mx_decode_f32<FMT, 1>(reg[p], power);
      } else if (p & 1) {
        lo = mx_decode_f32<FMT, 2>(reg[p / 2], power);
        hi = mx_decode_f32<FMT, 3>(reg[p / 2], power);
      } else {
        lo = mx_decode_f32<FMT, 0>(reg[p / 2], power);
        hi = mx_decode_f32<FMT, 1>(reg[p / 2], power);
      }
      x = u32x4{__float_as_uint(lo.x), __float_as_uint(lo.y), __float_as_uint(hi.x), __float_as_uint(hi.y)};
    }
    return x;
  }
  // Rows of an LDS tile from the place of load 0's unit, or of its own, to that of load i's.
  __device__ __forceinline__ static int rows_to(int i) { return i / GL * GROWS + (WHOLE ? i % GL * RPL : 0); }
  __device__ __forceinline__ void store_k(unsigned char *tile, int i) const {
    const int l = i / PIECES, p = i % PIECES;
    *reinterpret_cast<u32x4 *>(tile + k_lds[WHOLE ? 0 : l % GL] + rows_to(l) * C::KROWB + p * 16) = piece(k_reg[l], k_exp[l][0], p);
  }
  __device__ __forceinline__ void store_v(unsigned char *tile, int i) const {
    const int l = i / PIECES, p = i % PIECES;
    *reinterpret_cast<u32x4 *>(tile + v_lds[WHOLE ? 0 : l % GL] + rows_to(l) * C::VROWB + p * 16) = piece(v_reg[l], v_exp[l][0], p);
  }
  __device__ __forceinline__ void store(unsigned char *k_tile, unsigned char *v_tile) const {
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) store_k(k_tile, i);
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) store_v(v_tile, i);
  }
};

// N bytes of codes from the lane's place `at` on, the second 16 of 32 from `then` on.
template <int N, int POLICY>
__device__ __forceinline__ void load_units(const Buffer<POLICY> &from, unsigned (&to)[N / 4], unsigned at, unsigned then) {
  if constexpr (N <= 16) {
    from.template load<N>(to, at, 0);
  } else {
    static_assert(N == 32, "two loads");
    const u32x4 x = from.load16(at, 0), y = from.load16(then, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = x[i], to[4 + i] = y[i];
  }
}
// Codes 8 i .. 8 i + 7 of a lane's words as bf16.
template <int FMT, int W>
__device__ __forceinline__ u32x4 eight(const unsigned (&word)[W], float power, int i) {
  if constexpr (FMT == PF_MX_E4M3)
    return u32x4{mx_decode_bf16<FMT, 0>(word[2 * i], power), mx_decode_bf16<FMT, 1>(word[2 * i], power), mx_decode_bf16<FMT, 0>(word[2 * i + 1], power),
                 mx_decode_bf16<FMT, 1>(word[2 * i + 1], power)};
  else
    return u32x4{mx_decode_bf16<FMT, 0>(word[i], power), mx_decode_bf16<FMT, 1>(word[i], power), mx_decode_bf16<FMT, 2>(word[i], power),
                 mx_decode_bf16<FMT, 3>(word[i], power)};
}
// Over the four lanes l, l + 16, l + 32, l + 48; all get the result.
template <typename F>
__device__ __forceinline__ float over_groups(float v, F &&op) {
  const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = op(__uint_as_float(x[0]), __uint_as_float(x[1]));
  const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

// The few kernel: up to 16 rows of bf16 (tokens of a sequence times the query heads of a key head) over the keys, which are the work.
//   S^T[key][row] = K Q^T    in matrix instructions of 16 keys x 16 rows x 32 channels: a lane's K operand are channels of one key, which it
//                            loads and decodes itself.  Channel order is free as long as Q has the same: where a row is a multiple of 64
//                            channels the four lanes of a key hold a quarter of it each, one after the other, so that they load whole units.
//   O^T[c][row] += V^T P^T   V through LDS, decoded on its way there and read transposed; P^T are the scores' accumulators as they are, the weights
//                            rounded to bf16 for the matrix units (half a step of 2^-8 each, as in the kernels of attn_rows.h); their sum is of 32 bits.
// Against 32 rows it has half the accumulators, half the exponentials per key and, with K out of LDS, half the LDS: three or four
// workgroups fit a CU instead of two.  As in the key kernel every wave walks a quarter of the workgroup's keys in tiles of its own, and the
// loads of the next tile run meanwhile.
//   64 tokens over 190817 keys in all, 8 heads of 128, in a graph over three such caches, join included: e4m3 404 MB in 104 us against 120 in the key
//   kernel (alone, some of the keys still in the Infinity Cache, 83: 4.9 TB/s), e2m1 209 MB in 61 against 110.  Heads of 64: 54 - 59 and 43 us against
//   74 and 70, of 72 (16 of them) 165 and 128 against 178 and 138.
// In 8 bits it is bound by memory.  In 4 bits by latency: 2 to 3 waves to a SIMD, its vector unit busy for a third of the time.  Head sizes of 72 to 96 load
// K by 8 or 4 bytes, with an exponent for each, and two workgroups fit a CU: 2.7 and 1.8 TB/s at 72, 3.3 and 2.3 at 96.
constexpr int FEW_ROWS = 16;
constexpr int few_workgroups_of(int dhp) { return dhp == 64 ? 4 : dhp == 96 ? 2 : 3; }   // on a CU, by their registers
template <int DHP>
struct FewTile {
  static constexpr int WAVES = 4, TK = 32, RW = 32, ROWS = FEW_ROWS;
  static constexpr int ROWB = DHP * 2, KROWB = ROWB;
  static constexpr int VROWB = ROWB + 32;                          // an odd number of 32 bytes: those of 8 rows lie in different banks
  static constexpr int LOADS = RW * ROWB / 1024;
  static constexpr int POLICY = 2;                                 // every key is read once
  static constexpr int VTILE_B = TK * VROWB, OSTR = DHP + 4, JOIN_B = WAVES * ROWS * (OSTR + 2) * 4;
  static constexpr int SMEM = WAVES * VTILE_B > JOIN_B ? WAVES * VTILE_B : JOIN_B;
};
// The work of the few kernel: items of a row tile and a chunk of `chunk` keys each, sequence after sequence; one of no keys for a tile
// whose sequence has none.  Only the device knows how many there are, so the workgroups of a key head take them in turn, and none is
// launched for a chunk that is not there.  Lane i counts those of sequence i of a block of 64; an item's sequence is the number of lanes that end in
// front of it.
template <bool CAUSAL>
__device__ __forceinline__ void few_sequence(const RowsAttn &a, int s, int &q0, int &n, int &keys, int64_t &first) {
  int q1;
  sequence_rows(a.cu_q, s, a.total_q, q0, q1);
  n = q1 - q0;
  keys = clampi(a.kv_len[s], 0, a.pages.max_pages << a.pages.page_shift);
  first = CAUSAL ? a.first[s] : 0;
  if (CAUSAL) keys = (int)min((int64_t)keys, max(first + n, (int64_t)0));   // that its last row sees
}
__device__ __forceinline__ int few_chunks(int keys, int chunk) { return max((int)(((unsigned)keys + chunk - 1) / (unsigned)chunk), 1); }
template <bool CAUSAL>
__device__ __forceinline__ int few_ends(const RowsAttn &a, int group, int chunk, int block, int lane) {
  int end = 0;
  if (block + lane < a.n_seqs) {
    int q0, n, keys;
    int64_t first;
    few_sequence<CAUSAL>(a, block + lane, q0, n, keys, first);
    end = (n * group + FEW_ROWS - 1) / FEW_ROWS * few_chunks(keys, chunk);
  }
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int before = __shfl_up(end, o, kWave);
    end += lane >= o ? before : 0;
  }
  return end;
}
// Item number `at` of the block.
template <bool CAUSAL>
__device__ __forceinline__ void few_item(const RowsAttn &a, int group, int chunk, int block, int ends, int at, Work &w, int &all_chunks) {
  const int i = __builtin_popcountll(__builtin_amdgcn_ballot_w64(ends <= at));
  const int start = i == 0 ? 0 : __builtin_amdgcn_readlane(ends, i - 1);
  w.s = block + i;
  w.k0 = 0;
  int keys;
  few_sequence<CAUSAL>(a, w.s, w.q0, w.n, keys, w.first);
  all_chunks = few_chunks(keys, chunk);
  const int tiles = (w.n * group + FEW_ROWS - 1) / FEW_ROWS;
  w.sp = (at - start) / tiles;         // tiles of a chunk one after the other: they read the same keys
  w.r_first = (at - start - w.sp * tiles) * FEW_ROWS;
  w.k_end = keys;
  if (CAUSAL) w.k_end = (int)max(min((int64_t)keys, w.first + (min(w.r_first + FEW_ROWS, w.n * group) - 1) / group + 1), (int64_t)0);
  w.kb = (int)min((int64_t)w.k_end, (int64_t)w.sp * chunk);
  w.ke = (int)min((int64_t)w.k_end, (int64_t)(w.sp + 1) * chunk);
  w.zone = CAUSAL ? (int)max(min((int64_t)w.ke, w.first + w.r_first / group + 1), (int64_t)0) : w.ke;
}

// A kernel's arguments where the compiler does not know that they are the ones it has read before.
template <typename A>
__device__ __forceinline__ const A &again(const A &args) {
#if defined(__HIP_DEVICE_COMPILE__)
  auto at = (const __attribute__((address_space(4))) A *)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return *(const A *)at;
#else
  return args;
#endif
}

template <int DHP, int SRC, bool CAUSAL>
__global__ __launch_bounds__(256, (few_workgroups_of(DHP))) void attn_rows_few_kernel(RowsKernelArgs args) {
  using T = bf16_t;
  using C = FewTile<DHP>;
  using Loader = MxTileLoader<C, T, SRC>;
  constexpr int FMT = Loader::FMT, BITS = Loader::BITS, TK = C::TK, KS = DHP / 32, CB = DHP / 16;
  // K: PER neighbouring channels to a lane and load: all of its KS * 8, or 8 for each step
  constexpr bool WHOLE = DHP % 64 == 0;
  constexpr int PER = WHOLE ? KS * 8 : 8, KLOADS = WHOLE ? 1 : KS, KBYTES = PER * BITS / 8, KWORDS = KBYTES / 4;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  __shared__ unsigned hidden_all[C::WAVES][(C::ROWS + TK - 2) / TK + 1];
  const int kv_heads = args.a.kv_heads, slots = args.slots, most_items = args.most_items;
  const int hk = blockIdx.x % kv_heads;
  const int chunk = args.a.least_keys;
  int block = 0, ends = few_ends<CAUSAL>(args.a, args.group, chunk, 0, lane);
  int base = 0;                      // items in front of the block
  for (int item = blockIdx.x / kv_heads; item < most_items; item += slots) {
    while (item >= base + __builtin_amdgcn_readlane(ends, 63)) {
      base += __builtin_amdgcn_readlane(ends, 63);
      block += 64;
      if (block >= args.a.n_seqs || base >= most_items) return;
      ends = few_ends<CAUSAL>(args.a, args.group, chunk, block, lane);
    }
    const RowsKernelArgs &p = again(args);   // read again for every item: kept over all of them they cost more registers than there are
    const RowsAttn &a = p.a;
    const int dh = a.head_dim, G = p.group;
    Work w;
    int all_chunks;
    few_item<CAUSAL>(a, G, chunk, block, ends, item - base, w, all_chunks);
    w.hk = hk;
    const auto share = [&](int v, int &b, int &e) __attribute__((always_inline)) {   // wave v's keys
      const int q = ((w.ke - w.kb + C::WAVES - 1) / C::WAVES + TK - 1) / TK * TK;
      b = min(w.ke, w.kb + v * q);
      e = min(w.ke, b + q);
    };
    int kb, ke;
    share(wave, kb, ke);
    kb = uniform(kb);
    ke = uniform(ke);
    const int tiles = (ke - kb + TK - 1) / TK;

    const LaneRow row(w, G, l16);
    int limit = ke;                    // keys before this one are seen
    if (CAUSAL && row.ok && w.first + row.tok + 1 < limit) limit = w.first + row.tok + 1 < 0 ? 0 : (int)(w.first + row.tok + 1);
    int least = limit;
    for (int o = 8; o > 0; o >>= 1) least = min(least, __shfl_xor(least, o, kWave));
    least = uniform(least);

    const auto channel = [&](int ks) __attribute__((always_inline)) { return WHOLE ? g * PER + ks * 8 : ks * 32 + g * 8; };   // first of the lane's eight of step ks
    u32x4 qf[KS];
    {
      const T *qp = (const T *)a.q + (int64_t)(w.q0 + row.tok) * a.ldq + (int64_t)row.head * dh;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[ks] = u32x4{0, 0, 0, 0};
        if (row.ok && channel(ks) < dh) qf[ks] = *reinterpret_cast<const u32x4 *>(qp + channel(ks));
      }
    }

    Loader ld(a, w, lane, 0, kb, ke);
    unsigned k_reg[2][KLOADS][KWORDS], k_exp[2][KLOADS][1];
    unsigned k_off[KLOADS], k_then[KLOADS], k_exp_off[KLOADS];
#pragma unroll
    for (int i = 0; i < KLOADS; ++i) {
      const int c = channel(i), byte = c * BITS / 8;
      unsigned at = l16 * a.mx.row_bytes + byte, exp_at = l16 * a.mx.blocks + c / PF_MX_BLOCK;
      k_off[i] = byte < a.mx.row_bytes ? at : Loader::kOutside;
      k_then[i] = byte + 16 < a.mx.row_bytes ? at + 16 : Loader::kOutside;   // the next row's codes are not this one's, whatever Q has there
      k_exp_off[i] = byte < a.mx.row_bytes ? exp_at : Loader::kOutside;
    }
    const auto load = [&](int t) __attribute__((always_inline)) {
      ld.aim(t);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const Buffer<C::POLICY> codes(ld.k_from[b], ld.in_group[b] * a.mx.row_bytes), exps(ld.ks_from[b], ld.in_group[b] * a.mx.blocks);
#pragma unroll
        for (int i = 0; i < KLOADS; ++i) {
          load_units<KBYTES>(codes, k_reg[b][i], k_off[i], k_then[i]);
          exps.template load<1>(k_exp[b][i], k_exp_off[i], 0);
        }
      }
#pragma unroll
      for (int i = 0; i < C::LOADS; ++i) ld.load_v(i);
    };

    // keys with infinities or NaN among those that some row does not see
    constexpr int ZONE = (C::ROWS + TK - 2) / TK + 1;
    unsigned *const hidden = hidden_all[wave];
    const bool zoned = CAUSAL && w.zone < ke;
    const int zone_tile = zoned && w.zone > kb ? (w.zone - kb) / TK : 0;
    if (CAUSAL && lane < ZONE) hidden[lane] = 0;

    f32x4 o[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) o[cb] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;    // running maximum of the raw scores; the lane's share of the sum
    unsigned char *const tile = smem + wave * C::VTILE_B;
    const unsigned char *const v_at = tile + (4 * g + (l16 >> 2)) * C::VROWB + (l16 & 3) * 8;

    if (tiles > 0) load(0);
    for (int t = 0; t < tiles; ++t) {
      const unsigned groups = ld.groups;
      const bool clear = zoned && t >= zone_tile;
      if (uniform((int)clear) != 0) ld.clear_v(hidden, t - zone_tile);
#pragma unroll
      for (int i = 0; i < C::LOADS; ++i) ld.store_v(tile, i);
      __builtin_amdgcn_sched_barrier(0);   // here and below: what the next part needs is not brought in early, at the cost of registers
      f32x4 sc[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        sc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          const int i = WHOLE ? 0 : ks;
          const u32x4 kf = eight<FMT>(k_reg[b][i], mx_power(k_exp[b][i][0]), WHOLE ? ks : 0);
          sc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[ks]), sc[b], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (t + 1 < tiles) load(t + 1);
      const int key0 = kb + t * TK;
      if (key0 + TK > least || groups != Loader::kAllGroups) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (key0 + b * 16 + g * 4 + i >= limit || !((groups >> b) & 1)) sc[b][i] = -INFINITY;
      }
      float tmax = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])), fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
      tmax = over_groups(tmax, [](float x, float y) { return fmaxf(x, y); });
      const float m_new = fmaxf(m_run, tmax);
      const float m_use = m_new == -INFINITY ? 0.f : m_new;           // a row that has seen no key yet: weights 2^-inf = 0
      const float alpha = __builtin_amdgcn_exp2f((m_run - m_use) * p.sl2);
      const float neg = -m_use * p.sl2;
      m_run = m_new;
      float sum = 0.f;
      bf16x8 pf;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = __builtin_amdgcn_exp2f(fmaf(sc[e >> 2][e & 3], p.sl2, neg));
        sum += x;
        pf[e] = (bf16_t)x;
      }
      l_run = l_run * alpha + sum;
      if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {          // no rescale where no row's maximum moved
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[cb][i] *= alpha;
      }
      __builtin_amdgcn_sched_barrier(0);
      // place e of a lane's eight keys: key 4 g + (e & 3) of the first or second 16, the order in which the accumulators hold the weights
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        struct { s16x4 lo, hi4; } v8 = {lds_read_transposed(v_at + cb * 32), lds_read_transposed(v_at + 16 * C::VROWB + cb * 32)};
        o[cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v8), pf, o[cb], 0, 0, 0);
      }
    }
    float l_tot = over_groups(l_run, [](float x, float y) { return x + y; });

    // join the waves: each leaves (m, l, O), and sums a quarter of the channels in the waves' order
    __syncthreads();
    float *om = reinterpret_cast<float *>(smem), *ml = om + C::WAVES * C::ROWS * C::OSTR;
    float *mine = om + (wave * C::ROWS + l16) * C::OSTR;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) *reinterpret_cast<f32x4 *>(mine + cb * 16 + g * 4) = o[cb];
    if (g == 0) {
      ml[(wave * C::ROWS + l16) * 2] = m_run;
      ml[(wave * C::ROWS + l16) * 2 + 1] = l_tot;
    }
    __syncthreads();
    float m_all = -INFINITY;
#pragma unroll
    for (int v = 0; v < C::WAVES; ++v) m_all = fmaxf(m_all, ml[(v * C::ROWS + l16) * 2]);
    const float m_use = m_all == -INFINITY ? 0.f : m_all;
    float wt[C::WAVES];
    l_tot = 0.f;
#pragma unroll
    for (int v = 0; v < C::WAVES; ++v) {
      wt[v] = __builtin_amdgcn_exp2f((ml[(v * C::ROWS + l16) * 2] - m_use) * p.sl2);
      l_tot += wt[v] * ml[(v * C::ROWS + l16) * 2 + 1];
    }
    if (row.ok) {
      const float inv = l_tot != 0.f ? 1.f / l_tot : 0.f;
#pragma unroll
      for (int i = 0; i < (CB + 3) / 4; ++i) {
        const int c = (wave + C::WAVES * i) * 16 + g * 4;            // the lane's channels c .. c + 3
        if (c < dh) {
          f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int v = 0; v < C::WAVES; ++v) {
            const f32x4 x = *reinterpret_cast<const f32x4 *>(om + (v * C::ROWS + l16) * C::OSTR + c);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = fmaf(wt[v], x[e], acc[e]);
          }
          put4<T>(a, w.sp, w.q0 + row.tok, row.head, c, inv, acc[0], acc[1], acc[2], acc[3]);
        }
      }
      if (g == 0 && wave == 0) put_stats(a, w.sp, w.q0 + row.tok, row.head, m_all * p.sl2, l_tot);
    }
    // the tile's last chunk says of those that are not there that they are empty
    if (a.splits > 1 && w.sp == all_chunks - 1) {
      for (int i = threadIdx.x; i < (a.splits - all_chunks) * C::ROWS; i += 256) {
        const LaneRow empty(w, G, i % C::ROWS);
        if (empty.ok) put_stats(a, all_chunks + i / C::ROWS, w.q0 + empty.tok, empty.head, -INFINITY, 0.f);
      }
    }
    if (CAUSAL && w.zone < w.ke) {
#pragma unroll 1
      for (int v = 0; v < C::WAVES; ++v) {
        int b, e;
        share(v, b, e);
        if (w.zone < e) add_hidden<C, T, SRC, C::ROWS, 256>(p, w, hidden_all[v], ZONE, b + (w.zone > b ? (w.zone - b) / TK : 0) * TK, e);
      }
    }
    __syncthreads();                   // the next item's tiles take the LDS
  }
}

template <int DHP, int SRC, bool CAUSAL>
hipError_t launch_few(const RowsAttn &a, hipStream_t s) {
  using C = FewTile<DHP>;
  if (hipError_t e = allow_dynamic_lds<&attn_rows_few_kernel<DHP, SRC, CAUSAL>, C::SMEM>(); e != hipSuccess) return e;
  RowsKernelArgs p{a, a.n_heads / a.kv_heads, 0, a.scale * kLog2e};
  // so many workgroups as are resident at a time, or as there can be items
  p.most_items = (int)(((int64_t)a.total_q * p.group / C::ROWS + a.n_seqs) * a.splits);   // less than 2^25 by the caller's limit, in chunks 2^17 by the plan's
  const int resident = 256 * few_workgroups_of(DHP);
  p.slots = std::min(p.most_items, std::max(resident / a.kv_heads, 1));
  attn_rows_few_kernel<DHP, SRC, CAUSAL><<<dim3((unsigned)(p.slots * a.kv_heads)), 256, C::SMEM, s>>>(p);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || a.splits == 1 ? e : launch_rows_join(a, s);
}
template <int SRC, bool CAUSAL>
hipError_t launch_few_dim(const RowsAttn &a, hipStream_t s) {
  if (a.head_dim <= 64) return launch_few<64, SRC, CAUSAL>(a, s);
  if (a.head_dim <= 96) return launch_few<96, SRC, CAUSAL>(a, s);
  return launch_few<128, SRC, CAUSAL>(a, s);
}

template <typename T, int SRC>
hipError_t launch_mask(const RowsAttn &a, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (a.shape == ROWS_FEW) return a.causal ? launch_few_dim<SRC, true>(a, s) : launch_few_dim<SRC, false>(a, s);
  }
  return a.causal ? launch_dim<T, SRC, true>(a, s) : launch_dim<T, SRC, false>(a, s);
}

}  // namespace

RowsPlan mx_attention_plan(int dt, int format, int total_q, int n_seqs, int n_heads, int kv_heads, int head_dim, int64_t max_kv) {
  // Where a sequence has more rows than a tile of the few kernel its keys are read again: against the key kernel's tiles of 32 rows that is dearer in 8
  // bits (16 sequences of 20 rows over 8192 keys of 8 heads of 128: 121 us and 84) and not in 4 (70 and 71; of 32 rows 65 and 89).  In 8 bits one long
  // sequence among short ones costs, too (63 of 4 rows and one of 400: 306 us and 250, in 4 bits 173 and 205).  The totals do not show it; they are
  // taken for sequences of as many tokens each where they could be (16 of 16 rows: 76 and 84), and for such a mixture else.  Where a mixture's total happens to
  // divide it is taken wrongly (63 of 4 rows and one of 772: 330 us, of 760 in the key kernel 246).
  const bool alike = total_q <= n_seqs || total_q % n_seqs == 0;
  const int64_t rows = (int64_t)total_q * (n_heads / kv_heads), few = format == PF_MX_E2M1 ? 32 : alike ? 16 : 8;
  if (dt != DT_BF16 || rows > n_seqs * few) return rows_attention_plan(dt, total_q, n_seqs, n_heads, kv_heads, head_dim, max_kv);
  // Keys to a chunk.  All of them where they are few, or few enough with a tile for every CU (64 tokens over 1000 keys each, 8 / 4 bits: whole 35 / 21 us,
  // chunks of 512 40 / 27, of 256 43 / 30; over 2500 75 / 43, chunks of 1024 83 / 49).  Else 1024, which workgroups taking them in turn spread
  // evenly over caches of different lengths (64 tokens over up to 16384 keys 105 / 62, chunks of 512 111 / 69, of 2048 111 / 67); down to 256 with fewer
  // tiles (8 tokens over up to 8192 keys 18 with 256 or 512, 21 with 1024; one over 4096 13.1 with 256, 16.6 with 512).
  const int64_t w = workgroups(total_q, n_heads / kv_heads, n_seqs, kv_heads, 16);
  int64_t c = w >= 256 ? 1024 : std::min(std::max(w * max_kv / 2048, (int64_t)256), (int64_t)1024);
  if (max_kv <= (w >= 256 ? 2560 : 512)) c = max_kv;
  // The host knows how long a cache could be, not how long it is: chunks that are not there cost the join a read each, and all of them their place in the
  // workspace.  With at most 65536 items (partial results of 16 rows) a wide table costs neither: 1024 tokens over 1000 / 4000 keys each in one for 131072 keys,
  // 8 bits, take 452 / 1441 us and 136 MB of workspace, without the bound 882 / 2214 and 2.2 GB.  Less is better for caches of one length (8192 items: 384 /
  // 1359) and worse where a few are long (24 heads of 64, 64 tokens over up to 16384 keys in the same table: 141 us, 32768 items 193, 8192 items 240).
  const int64_t most = std::max(65536 / w, (int64_t)1);
  c = std::max(c, std::max((max_kv + most - 1) / most, (max_kv + kMaxChunks - 1) / kMaxChunks));
  c = (c + 127) / 128 * 128;
  RowsPlan p{ROWS_FEW, (int)((max_kv + c - 1) / c), (int)c, 0};
  if (p.splits > 1) p.ws_bytes = (size_t)p.splits * total_q * n_heads * (head_dim + 2) * sizeof(float);
  return p;
}

hipError_t launch_mx_attention(const RowsAttn &a, hipStream_t s) {
  if (a.dt == DT_BF16) return a.mx.format == PF_MX_E4M3 ? launch_mask<bf16_t, KEYS_E4M3>(a, s) : launch_mask<bf16_t, KEYS_E2M1>(a, s);
  return a.mx.format == PF_MX_E4M3 ? launch_mask<float, KEYS_E4M3>(a, s) : launch_mask<float, KEYS_E2M1>(a, s);
}

}  // namespace pf
