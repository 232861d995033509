// Attention of packed rows over pages of 8- or 4-bit numbers: the kernels of attn_rows.h with a loader that brings codes from memory and
// writes what they stand for to LDS, in the type of the rows.
//
// Every value that the pages can hold is a number of both types, so from the LDS on nothing differs from pages of rows, and the
// results are bit for bit those over pages that hold the decoded rows.  A tile needs half or a quarter of the bytes from memory, and a
// conversion instruction for two channels on its way to LDS.
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

template <typename T, int SRC>
hipError_t launch_mask(const RowsAttn &a, hipStream_t s) {
  return a.causal ? launch_dim<T, SRC, true>(a, s) : launch_dim<T, SRC, false>(a, s);
}

}  // namespace

hipError_t launch_mx_attention(const RowsAttn &a, hipStream_t s) {
  if (a.dt == DT_BF16) return a.mx.format == PF_MX_E4M3 ? launch_mask<bf16_t, KEYS_E4M3>(a, s) : launch_mask<bf16_t, KEYS_E2M1>(a, s);
  return a.mx.format == PF_MX_E4M3 ? launch_mask<float, KEYS_E4M3>(a, s) : launch_mask<float, KEYS_E2M1>(a, s);
}

}  // namespace pf
