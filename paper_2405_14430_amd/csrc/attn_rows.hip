// Attention of packed query rows over packed keys or over pages (gfx950 matrix instructions, 32-bit softmax and sums).
//
// out_i = sum_j softmax_j(scale q_i . k_j) v_j in one pass over the keys with a running maximum and sum:
//   S^T[key][row] = K[key][:] . Q[row][:]        A = K tile (LDS), B = Q fragments (registers)
//   O^T[c][row]  += V^T[c][key] . P^T[key][row]  A = V tile (LDS, read transposed), B = P^T, the S^T accumulators as they are
// so that a lane owns one row: the softmax is in-lane but for one exchange between the half-waves.
//
// A "row" is a (token, head) pair of one key head: the G = n_heads / kv_heads query heads that share a key head are packed
// behind each other, token by token, and a K / V tile that is loaded serves all of them.  A wave holds 32 rows.
//   tile kernel (KW = 1): NW waves of 32 rows each share tiles of 64 keys (fp32: 32);
//   key kernel  (KW = 4): four waves hold the same 32 rows and each walks a quarter of the keys in tiles of its own, without
//                         a barrier; they are joined through LDS at the end.  For few rows per sequence, where the keys
//                         are the work.
//   wide kernel (bf16):   four waves of 64 rows, below.
// The keys of a launch with few workgroups are cut into chunks, whose partial results a second launch joins.
//
// What bounds them, and what they measured.  Wide: the matrix cores and the power they take: six causal prompts (28223 rows
// of 32 heads of 128 over 8 key heads) 2.38 - 2.45 ms, 1.15 - 1.19 PFLOP/s (a library product of 8192 cubed: 1.42); at head sizes up to 80 the vector
// unit more, an exponential, a multiply-add and an add per score: 22256 rows of 16 heads of 72 in six images 0.68 - 0.71 ms, 0.83 - 0.86 PFLOP/s.  Keys: memory: 64 tokens of 32
// heads of 128 over caches of up to 16384 keys of 8 heads 150 us, 783 MB at 5.2 TB/s; one token over 131072 keys of two heads 30 us, 5 of
// them the join's.  Tiles: the LDS (every MFMA takes a fragment from it) and, in fp32, the matrix cores: 4096 rows of 16 heads of 64 0.54 ms,
// 126 TFLOP/s (a library product of 4096 cubed: 138).
//
// Scores, their exponentials, the running maximum, the denominators and the outputs' sums are in 32 bits.  For bf16 rows the weights are rounded to
// bf16 for the second product, because the matrix units take both operands in one type and multiply fp32 at a tenth of the rate; the
// denominator sums them unrounded, which is what the log-sum-exp needs.  Against 64 bits the output's relative error grows from the 0.0017 of its own
// rounding to 0.0023 at most (0.0021 for single tokens).
//
// Tiles come from memory through registers: while the products of tile t run, the loads of tile t + 1 are in flight.  The
// bounds of the buffer loads give zeros for rows past the last key, for pages that are none and for channels past the head, so
// neither the scores nor 0 * v meets what lies there.  LDS rows are padded against bank conflicts.
#include <algorithm>
#include <type_traits>

#include "requests.h"

namespace pf {
namespace {

// f(integral_constant<int, 0>) ... f(integral_constant<int, N - 1>), in order
template <int N, int I = 0, typename F>
__device__ __forceinline__ void unrolled(F &&f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    unrolled<N, I + 1>(f);
  }
}

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxChunks = 256;
constexpr float kLn2 = 0.6931471805599453f;

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

#if defined(__HIP_DEVICE_COMPILE__)
template <int POLICY>
struct Buffer {   // `bytes` bytes from a wave-uniform address; loads past them give zeros
  __amdgpu_buffer_rsrc_t rs;
  __device__ __forceinline__ Buffer(const void *base, unsigned bytes)
      : rs(__builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, bytes, 0x00020000)) {}
  __device__ __forceinline__ u32x4 load16(unsigned lane_at, unsigned at) const {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, lane_at, at, POLICY));
  }
};
__device__ __forceinline__ s16x4 lds_read_transposed(const unsigned char *p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p);
}
#else   // the host pass only parses the kernels
template <int POLICY>
struct Buffer {
  __device__ Buffer(const void *, unsigned) {}
  __device__ u32x4 load16(unsigned, unsigned) const { return u32x4{}; }
};
__device__ s16x4 lds_read_transposed(const unsigned char *) { return s16x4{}; }
#endif

// A pointer or number that all lanes agree on, in scalar registers.
template <typename T>
__device__ __forceinline__ const T *uniform(const T *p) {
  const uint64_t u = (uint64_t)p;
  return (const T *)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)u));
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

struct RowsKernelArgs {
  RowsAttn a;
  int group;        // query heads per key head
  int slots;        // row tiles the grid has per key head
  float sl2;        // scale * log2(e)
};

template <typename T, int DHP, int NW_, int KW_>
struct Tile {
  static constexpr bool F32 = sizeof(T) == 4;
  static constexpr int NW = NW_, KW = KW_;
  static constexpr int WAVES = NW * KW;
  static constexpr int TK = NW > 1 && !F32 ? 64 : 32;      // keys per tile
  static constexpr int NB = TK / 32;                       // blocks of 32 keys
  static constexpr int CB = DHP / 32;                      // blocks of 32 channels
  static constexpr int ROWB = DHP * (int)sizeof(T);        // bytes of an LDS row
  // LDS rows are padded so that what is read together lies in different banks: K as 16 bytes of 16 rows (16 bytes further a
  // row), V as 64 bytes of four rows (bf16, transposed: 64 bytes further modulo 256) or 128 bytes of rows r and r + 4 (fp32)
  static constexpr int KROWB = ROWB + 16;
  static constexpr int VROWB = F32 ? ROWB + 32 : ROWB % 256 == 192 ? ROWB : ROWB + 64;
  static constexpr int KTILE_B = TK * KROWB, VTILE_B = TK * VROWB;
  static constexpr int RW = TK / NW;                       // rows of a tile that one wave brings in
  static constexpr int LOADS = RW * ROWB / 1024;           // its 1 KB loads
  static constexpr int BUFS = NW > 1 ? 2 : 1;
  // Where no sequence has more than 32 rows the key kernel reads every key once: non-temporal loads (policy bit 1) leave the caches to
  // what is read again (64 tokens over caches of up to 16k keys 191 -> 172 us).  It keeps them where the plan gives it more rows, whose tiles
  // share keys through the L2s (not measured without).  For the wide kernel's they cost time (2.33 -> 2.49 ms).
  static constexpr int POLICY = KW > 1 ? 2 : 0;
  static constexpr int JOIN_B = KW > 1 ? KW * 32 * (DHP + 4 + 2) * 4 : 0;   // the waves' partial results
  static constexpr int SMEM = KW * BUFS * (KTILE_B + VTILE_B) > JOIN_B ? KW * BUFS * (KTILE_B + VTILE_B) : JOIN_B;
  static constexpr int ROWS = 32 * NW;                     // query rows of a workgroup
  static constexpr int WGS = SMEM > 80 * 1024 ? 1 : 2;     // workgroups on a CU, by their LDS
};

// Keys of sequence s, inside what there is.
template <bool PAGED>
__device__ __forceinline__ int sequence_keys(const RowsAttn &a, int s, int &k0) {
  if constexpr (PAGED) {
    k0 = 0;
    return clampi(a.kv_len[s], 0, a.pages.max_pages << a.pages.page_shift);
  } else {
    int k1;
    sequence_rows(a.cu_k, s, a.total_k, k0, k1);
    return k1 - k0;
  }
}

// The rows and keys of a workgroup.  Workgroup id -> (key head, row tile, chunk): neighbouring ids are different key heads - ids go
// round the 8 XCDs, so with 8 or more key heads a head's workgroups meet in one L2 - and later row tiles, which see more
// keys, come first, all of one chunk before those of the next, whose last ones have no keys where sequences are shorter than the longest or
// than the launch could take.  Row tiles of sequence s are slots floor(cu[s] G / ROWS) + s and on: enough of them for any start.
struct Work {
  int hk, sp, s;
  int q0, n;              // the sequence's first row and its number of rows
  int r_first;            // first (token, head) row of the tile
  int k0, k_end;          // packed: row of key 0; keys that some row of the tile sees lie before k_end
  int kb, ke;             // the chunk's
  int64_t first;          // slot of query 0
  int zone;               // keys from here to ke are hidden from some row of the tile (ke: none are)
};
template <bool PAGED, bool CAUSAL, int ROWS, int UNIT>
__device__ __forceinline__ bool find_work(const RowsKernelArgs &p, int lane, Work &w) {
  const RowsAttn &a = p.a;
  const int G = p.group;
  const int rest = blockIdx.x / a.kv_heads;
  w.hk = blockIdx.x % a.kv_heads;
  w.sp = rest / p.slots;
  const int slot = p.slots - 1 - rest % p.slots;
  w.s = wave_search(a.n_seqs - 1, lane, slot, [&](int i) { return clampi(a.cu_q[i], 0, a.total_q) * G / ROWS + i; });
  if (w.s < 0) return false;
  int q1;
  sequence_rows(a.cu_q, w.s, a.total_q, w.q0, q1);
  w.n = q1 - w.q0;
  w.r_first = (slot - (w.q0 * G / ROWS + w.s)) * ROWS;
  if (w.r_first < 0 || w.r_first >= w.n * G) return false;
  const int kn = sequence_keys<PAGED>(a, w.s, w.k0);
  w.first = !CAUSAL ? 0 : PAGED ? a.first[w.s] : kn - w.n;
  const int t_last = (w.r_first + ROWS < w.n * G ? w.r_first + ROWS - 1 : w.n * G - 1) / G;
  w.k_end = kn;
  if (CAUSAL && w.first + t_last + 1 < w.k_end) w.k_end = w.first + t_last + 1 < 0 ? 0 : (int)(w.first + t_last + 1);
  w.kb = 0;
  w.ke = w.k_end;
  if (a.splits > 1) {
    // equal parts, in UNITs, of the longest sequence of the launch, at least the plan's
    int64_t c = a.least_keys;
    if (w.sp * c < w.k_end) {
      int longest = 0;
      for (int i = lane; i < a.n_seqs; i += 64) {
        int unused;
        longest = max(longest, sequence_keys<PAGED>(a, i, unused));
      }
      for (int o = 32; o > 0; o >>= 1) longest = max(longest, __shfl_xor(longest, o, kWave));
      const int units = (longest + UNIT - 1) / UNIT;
      c = max(c, (int64_t)((units + a.splits - 1) / a.splits) * UNIT);
    }
    w.kb = (int)min((int64_t)w.k_end, w.sp * c);
    w.ke = (int)min((int64_t)w.k_end, (w.sp + 1) * c);
  }
  w.zone = w.ke;
  if (CAUSAL && w.first + w.r_first / G + 1 < w.ke) w.zone = w.first + w.r_first / G + 1 < 0 ? 0 : (int)(w.first + w.r_first / G + 1);
  return true;
}

// (token, head) row `at` of a workgroup's tile.
struct LaneRow {
  bool ok;
  int tok, head;
  __device__ __forceinline__ LaneRow(const Work &w, int G, int at) {
    const int r = w.r_first + at;
    ok = r < w.n * G;
    tok = ok ? r / G : 0;
    head = w.hk * G + (ok ? r - tok * G : 0);
  }
};

// Brings a wave's RW rows (from row LW on) of K and V tiles of TK keys from memory into registers, and from there into LDS.  The rows
// of a load lie in one group of 16 keys, so in one page.
template <typename C, typename T, bool PAGED>
struct TileLoader {
  static constexpr int TK = C::TK, ROWB = C::ROWB;
  static constexpr int GROUPS = C::RW > 16 ? C::RW / 16 : 1;      // page groups a wave loads per tile
  static constexpr int GL = C::LOADS / GROUPS;                     // loads per group
  static constexpr int GROWS = C::RW / GROUPS;
  static constexpr int TPB = 1024 / TK;                            // tiles per block of 64 groups
  static constexpr unsigned kOutside = 0x7fff0000u;
  static constexpr unsigned kAllGroups = (1u << (TK / 16)) - 1;
  const RowsAttn &a;
  const int lane, lw, s, kb, ke;
  unsigned k_row, v_row;                                           // bytes between rows
  // The lane's bytes from a group's first row, and where they go in an LDS tile.  Where a load is a whole number of rows its
  // lanes' offsets are those of the first one, so many rows further.
  static constexpr bool WHOLE = 1024 % ROWB == 0;
  static constexpr int OFFS = WHOLE ? 1 : C::LOADS, RPL = 1024 / ROWB;
  unsigned k_off[OFFS], v_off[OFFS];
  int k_lds[OFFS], v_lds[OFFS];
  const T *k_head, *v_head;
  // Pages: lane i holds the page of 16-key group i of the current 1024 keys, and of the next 1024 (loaded that far ahead).
  int page_now = -1, page_next = -1;
  unsigned groups = kAllGroups;                                    // which groups of the tile in the registers have a page
  const T *k_from[GROUPS], *v_from[GROUPS];
  int in_group[GROUPS];                                            // rows of the group that there are
  u32x4 k_reg[C::LOADS], v_reg[C::LOADS];

  __device__ __forceinline__ TileLoader(const RowsAttn &args, const Work &w, int lane_, int lw_, int kb_, int ke_)
      : a(args), lane(lane_), lw(lw_), s(w.s), kb(kb_), ke(ke_) {
    const int dh = a.head_dim;
    k_row = (unsigned)((PAGED ? (int64_t)dh : a.ldk) * (int64_t)sizeof(T));
    v_row = (unsigned)((PAGED ? (int64_t)dh : a.ldv) * (int64_t)sizeof(T));
#pragma unroll
    for (int i = 0; i < OFFS; ++i) {
      const int off = i * 1024 + lane * 16, row = off / ROWB, byte = off % ROWB;
      k_off[i] = byte < dh * (int)sizeof(T) ? row % GROWS * k_row + byte : kOutside;
      v_off[i] = byte < dh * (int)sizeof(T) ? row % GROWS * v_row + byte : kOutside;
      k_lds[i] = (lw * C::RW + row) * C::KROWB + byte;
      v_lds[i] = (lw * C::RW + row) * C::VROWB + byte;
    }
    if constexpr (PAGED) {
      k_head = (const T *)a.pages.k + ((int64_t)w.hk << a.pages.page_shift) * dh;
      v_head = (const T *)a.pages.v + ((int64_t)w.hk << a.pages.page_shift) * dh;
      page_next = table_entry(0);
    } else {
      k_head = (const T *)a.k + (int64_t)w.k0 * a.ldk + (int64_t)w.hk * dh;
      v_head = (const T *)a.v + (int64_t)w.k0 * a.ldv + (int64_t)w.hk * dh;
    }
  }
  __device__ __forceinline__ int table_entry(int block) const {
    const int64_t key = (int64_t)kb + block * 1024 + lane * 16;
    int pg = -1;
    if (key < ke) pg = a.pages.table[(int64_t)s * a.pages.max_pages + (key >> a.pages.page_shift)];
    return pg >= 0 && pg < a.pages.n_pages ? pg : -1;
  }
  // Sets the sources of tile t's loads.  Tiles have to be taken in order, each once; tiles behind the last one read as zeros.
  __device__ __forceinline__ void aim(int t) {
    if constexpr (PAGED) {
      if (t % TPB == 0) {
        page_now = page_next;
        page_next = table_entry(t / TPB + 1);
      }
      groups = (unsigned)(__builtin_amdgcn_ballot_w64(page_now >= 0) >> ((t % TPB) * (TK / 16))) & kAllGroups;
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int key = kb + t * TK + lw * C::RW + g * GROWS;       // wave-uniform
      int rows = clampi(ke - key, 0, GROWS);
      if constexpr (PAGED) {
        const int pg = __builtin_amdgcn_readlane(page_now, (t % TPB) * (TK / 16) + ((lw * C::RW + g * GROWS) >> 4));
        if (pg < 0) rows = 0;
        const int64_t at = (int64_t)(key & ((1 << a.pages.page_shift) - 1)) * a.head_dim;
        k_from[g] = uniform(k_head + (pg < 0 ? 0 : pg * a.pages.k_stride + at));
        v_from[g] = uniform(v_head + (pg < 0 ? 0 : pg * a.pages.v_stride + at));
      } else {
        k_from[g] = uniform(k_head + (rows ? key * a.ldk : 0));
        v_from[g] = uniform(v_head + (rows ? key * a.ldv : 0));
      }
      in_group[g] = uniform(rows);
    }
  }
  // Values that the mask hides from some rows of the tile have weight 0 there, and 0 times an infinity or a NaN is none: for tiles with
  // such keys the V registers are cleared of them before they go to LDS, and the keys noted in `hidden` (one bit a
  // key; nearly always none).  `at`: the tile's place in `hidden`.
  __device__ __forceinline__ void clear_v(unsigned *hidden, int at) {
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) {
      bool bad = false;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        unsigned u = v_reg[i][e];
        if constexpr (sizeof(T) == 2) {
          if ((u & 0x7f80u) == 0x7f80u) { u &= 0xffff0000u; bad = true; }
          if ((u & 0x7f800000u) == 0x7f800000u) { u &= 0xffffu; bad = true; }
        } else {
          if ((u & 0x7f800000u) == 0x7f800000u) { u = 0; bad = true; }
        }
        v_reg[i][e] = u;
      }
      const int row = lw * C::RW + (i * 1024 + lane * 16) / ROWB;
      if (bad) atomicOr(hidden + at * (TK / 32) + (row >> 5), 1u << (row & 31));
    }
  }
  __device__ __forceinline__ void load_k(int i) {
    k_reg[i] = Buffer<C::POLICY>(k_from[i / GL], in_group[i / GL] * k_row).load16(k_off[WHOLE ? 0 : i], WHOLE ? i % GL * RPL * k_row : 0);
  }
  __device__ __forceinline__ void load_v(int i) {
    v_reg[i] = Buffer<C::POLICY>(v_from[i / GL], in_group[i / GL] * v_row).load16(v_off[WHOLE ? 0 : i], WHOLE ? i % GL * RPL * v_row : 0);
  }
  __device__ __forceinline__ void load(int t) {
    aim(t);
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) load_k(i);
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) load_v(i);
  }
  __device__ __forceinline__ void store_k(unsigned char *tile, int i) const { *reinterpret_cast<u32x4 *>(tile + k_lds[WHOLE ? 0 : i] + (WHOLE ? i * RPL * C::KROWB : 0)) = k_reg[i]; }
  __device__ __forceinline__ void store_v(unsigned char *tile, int i) const { *reinterpret_cast<u32x4 *>(tile + v_lds[WHOLE ? 0 : i] + (WHOLE ? i * RPL * C::VROWB : 0)) = v_reg[i]; }
  __device__ __forceinline__ void store(unsigned char *k_tile, unsigned char *v_tile) const {
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) store_k(k_tile, i);
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) store_v(v_tile, i);
  }
};

// One row's channels c .. c + 3 of the result, or of its partial result.
template <typename T>
__device__ __forceinline__ void put4(const RowsAttn &a, int sp, int64_t row, int head, int c, float inv, float x0, float x1, float x2, float x3) {
  if (a.splits > 1) {
    float *dst = a.ws + (((int64_t)sp * a.total_q + row) * a.n_heads + head) * a.head_dim + c;
    *reinterpret_cast<float4 *>(dst) = make_float4(x0, x1, x2, x3);
    return;
  }
  T *dst = (T *)a.out + row * a.ldo + (int64_t)head * a.head_dim + c;
  if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(dst) = make_float4(x0 * inv, x1 * inv, x2 * inv, x3 * inv);
  else *reinterpret_cast<bf16x4 *>(dst) = bf16x4{(bf16_t)(x0 * inv), (bf16_t)(x1 * inv), (bf16_t)(x2 * inv), (bf16_t)(x3 * inv)};
}
// m: the reference exponent (of 2) that l is relative to
__device__ __forceinline__ void put_stats(const RowsAttn &a, int sp, int64_t row, int head, float m, float l) {
  const int64_t at = row * a.n_heads + head;
  if (a.splits > 1) {
    float *dst = a.ws + (int64_t)a.splits * a.total_q * a.n_heads * a.head_dim + ((int64_t)sp * a.total_q * a.n_heads + at) * 2;
    *reinterpret_cast<float2 *>(dst) = make_float2(l != 0.f ? m : -INFINITY, l);
  } else if (a.lse) {
    a.lse[at] = l != 0.f ? m * kLn2 + logf(l) : -INFINITY;
  }
}

// A chunk without keys leaves its rows' statistics only; its partial results are not read.
template <int ROWS>
__device__ __forceinline__ bool empty_chunk(const RowsKernelArgs &p, const Work &w) {
  if (p.a.splits == 1 || w.kb < w.ke) return false;
  if (threadIdx.x < ROWS) {
    const LaneRow row(w, p.group, threadIdx.x);
    if (row.ok) put_stats(p.a, w.sp, w.q0 + row.tok, row.head, -INFINITY, 0.f);
  }
  return true;
}

// What the keys noted in `hidden` (n words, from key0 on; keys at ke and behind are none) bring to the rows that do see them: their
// infinities and NaN, whatever the weight, added to the rows that the workgroup has stored.  Nearly always there are none.
template <typename T, bool PAGED, int ROWS, int THREADS>
__device__ __forceinline__ void add_hidden(const RowsKernelArgs &p, const Work &w, const unsigned *hidden, int n, int key0, int ke) {
  const RowsAttn &a = p.a;
  unsigned any = 0;
  for (int i = 0; i < n; ++i) any |= hidden[i];
  if (__builtin_amdgcn_readfirstlane(any) == 0) return;
  __threadfence_block();
  __syncthreads();                        // every row is stored
  const int dh = a.head_dim;
  for (int i = 0; i < n; ++i)
    for (unsigned bits = hidden[i]; bits; bits &= bits - 1) {
      const int key = key0 + i * 32 + __builtin_ctz(bits);
      if (key >= ke) break;
      const T *v;
      if constexpr (PAGED) {
        const int pg = a.pages.table[(int64_t)w.s * a.pages.max_pages + (key >> a.pages.page_shift)];
        if (pg < 0 || pg >= a.pages.n_pages) continue;
        v = (const T *)a.pages.v + pg * a.pages.v_stride + (((int64_t)w.hk << a.pages.page_shift) + (key & ((1 << a.pages.page_shift) - 1))) * dh;
      } else {
        v = (const T *)a.v + (int64_t)(w.k0 + key) * a.ldv + (int64_t)w.hk * dh;
      }
      for (int e = threadIdx.x; e < ROWS * dh; e += THREADS) {
        const int r = w.r_first + e / dh, c = e % dh, tok = r / p.group;
        const float x = to_f32(v[c]);
        if (r >= w.n * p.group || key > w.first + tok || fabsf(x) <= 3.4028235e38f) continue;
        const int64_t row = w.q0 + tok, head = w.hk * p.group + r - tok * p.group;
        if (a.splits > 1) a.ws[(((int64_t)w.sp * a.total_q + row) * a.n_heads + head) * dh + c] += x;
        else ((T *)a.out)[row * a.ldo + head * dh + c] = from_f32<T>(to_f32(((T *)a.out)[row * a.ldo + head * dh + c]) + x);
      }
    }
}

template <typename T, int DHP, bool PAGED, bool CAUSAL, int NW, int KW>
__global__ __launch_bounds__(64 * NW * KW, (Tile<T, DHP, NW, KW>::WGS)) void attn_rows_kernel(RowsKernelArgs p) {
  using C = Tile<T, DHP, NW, KW>;
  constexpr int TK = C::TK, NB = C::NB, CB = C::CB;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const RowsAttn &a = p.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int l32 = lane & 31, hi = lane >> 5;
  const int dh = a.head_dim, G = p.group;
  Work w;
  if (!find_work<PAGED, CAUSAL, C::ROWS, 64 * KW>(p, lane, w)) return;   // chunks: whole tiles for all waves
  if (empty_chunk<C::ROWS>(p, w)) return;
  int kb = w.kb, ke = w.ke;
  if constexpr (KW > 1) {            // the wave's quarter
    const int q = ((ke - kb + KW - 1) / KW + TK - 1) / TK * TK;
    kb = min(ke, kb + wave * q);
    ke = min(ke, kb + q);
  }
  kb = __builtin_amdgcn_readfirstlane(kb);
  ke = __builtin_amdgcn_readfirstlane(ke);
  const int tiles = (ke - kb + TK - 1) / TK;

  // ---- the lane's row
  const LaneRow row(w, G, (KW > 1 ? 0 : wave) * 32 + l32);
  int limit = ke;                    // keys before this one are seen
  if (CAUSAL && row.ok && w.first + row.tok + 1 < limit) limit = w.first + row.tok + 1 < 0 ? 0 : (int)(w.first + row.tok + 1);
  int least = limit;                 // of all rows of the wave: tiles below it need no mask
  for (int o = 32; o > 0; o >>= 1) least = min(least, __shfl_xor(least, o, kWave));
  least = __builtin_amdgcn_readfirstlane(least);

  // ---- Q fragments: bf16: channels ks * 16 + 8 hi .. + 7; fp32: channels j * 8 + 4 hi .. + 3
  constexpr int NQ = C::F32 ? DHP / 8 : DHP / 16;
  u32x4 qf[NQ];
  {
    const T *qp = (const T *)a.q + (int64_t)(w.q0 + row.tok) * a.ldq + (int64_t)row.head * dh;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const int c = C::F32 ? i * 8 + hi * 4 : i * 16 + hi * 8;
      qf[i] = u32x4{0, 0, 0, 0};
      if (row.ok && c < dh) qf[i] = *reinterpret_cast<const u32x4 *>(qp + c);
    }
  }
  TileLoader<C, T, PAGED> ld(a, w, lane, KW > 1 ? 0 : wave, kb, ke);
  constexpr int BUF_B = C::KTILE_B + C::VTILE_B;
  unsigned char *const ring = smem + (KW > 1 ? wave * C::BUFS * BUF_B : 0);
  // keys with infinities or NaN among those that some row does not see: the zone spans fewer keys than the tile has rows
  constexpr int ZONE = (C::ROWS + TK - 2) / TK + 1;              // tiles it can touch
  __shared__ unsigned hidden_all[KW][ZONE * (TK / 32)];
  unsigned *const hidden = hidden_all[KW > 1 ? wave : 0];
  const bool zoned = CAUSAL && w.zone < ke;
  const int zone_tile = zoned && w.zone > kb ? (w.zone - kb) / TK : 0;
  if ((CAUSAL && KW > 1) || zoned) {
    if ((KW > 1 ? lane : (int)threadIdx.x) < ZONE * (TK / 32)) hidden[KW > 1 ? lane : threadIdx.x] = 0;
    if constexpr (NW > 1) __syncthreads();
  }
  auto store_tile = [&](int t) __attribute__((always_inline)) {
    if (zoned && t >= zone_tile) ld.clear_v(hidden, t - zone_tile);
    const int buf = t & (C::BUFS - 1);
    ld.store(ring + buf * BUF_B, ring + buf * BUF_B + C::KTILE_B);
  };

  f32x16 o[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[cb][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;    // running maximum of the raw scores; the lane's share of the sum

  // LDS addresses of the lane: K row l32; V, bf16: row 4 hi + (i >> 2), channels 16 g1 + 4 (i & 3) of a block; fp32: row 4 hi, channel l32
  const int i16 = lane & 15, g1 = (lane >> 4) & 1;
  const int k_at = l32 * C::KROWB + hi * 16;
  const int v_at = C::KTILE_B + (C::F32 ? 4 * hi * C::VROWB + l32 * 4 : (4 * hi + (i16 >> 2)) * C::VROWB + g1 * 32 + (i16 & 3) * 8);

  auto work_tile = [&](int t, int buf, unsigned groups) __attribute__((always_inline)) {
    const unsigned char *kt = ring + buf * BUF_B + k_at, *vt = ring + buf * BUF_B + v_at;
    f32x16 sc[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[b][i] = 0.f;
    if constexpr (!C::F32) {
#pragma unroll
      for (int ks = 0; ks < DHP / 16; ++ks)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(kt + b * 32 * C::KROWB + ks * 32);
          sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, __builtin_bit_cast(bf16x8, qf[ks]), sc[b], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int j = 0; j < DHP / 8; ++j) {
        const f32x4 kf = *reinterpret_cast<const f32x4 *>(kt + j * 32);
        const f32x4 qv = __builtin_bit_cast(f32x4, qf[j]);
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qv[e], sc[0], 0, 0, 0);
      }
    }
    const int key0 = kb + t * TK;
    if (key0 + TK > least || (PAGED && groups != ld.kAllGroups)) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = b * 32 + 8 * (i >> 2) + (i & 3);          // + 4 hi: the group of 16 is the same
          if (key0 + at + 4 * hi >= limit || (PAGED && !((groups >> (at >> 4)) & 1))) sc[b][i] = -INFINITY;
        }
    }
    float tmax = sc[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) tmax = fmaxf(tmax, sc[b][i]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(tmax), __float_as_uint(tmax), false, false);
    const float m_new = fmaxf(m_run, fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])));
    const float m_use = m_new == -INFINITY ? 0.f : m_new;           // a row that has seen no key yet: weights 2^-inf = 0
    const float alpha = __builtin_amdgcn_exp2f((m_run - m_use) * p.sl2);
    const float neg = -m_use * p.sl2;
    m_run = m_new;
    float sum = 0.f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        sc[b][i] = __builtin_amdgcn_exp2f(fmaf(sc[b][i], p.sl2, neg));
        sum += sc[b][i];
      }
    l_run = l_run * alpha + sum;
    if (__builtin_amdgcn_ballot_w64(alpha != 1.0f) != 0) {          // no rescale where no row's maximum moved
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[cb][i] *= alpha;
    }
    if constexpr (!C::F32) {
      // step j: keys 16 j + 4 hi + 0..3 and + 8: the order in which accumulators 8 (j % 2) .. + 7 hold their weights
#pragma unroll
      for (int j = 0; j < TK / 16; ++j) {
        bf16x8 pf;
#pragma unroll
        for (int e = 0; e < 8; ++e) pf[e] = (bf16_t)sc[j >> 1][8 * (j & 1) + e];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          struct { s16x4 lo, hi4; } v8 = {lds_read_transposed(vt + j * 16 * C::VROWB + cb * 64), lds_read_transposed(vt + (j * 16 + 8) * C::VROWB + cb * 64)};
          o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v8), pf, o[cb], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          const float vf = *reinterpret_cast<const float *>(vt + (8 * (i >> 2) + (i & 3)) * C::VROWB + cb * 128);
          o[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, sc[0][i], o[cb], 0, 0, 0);
        }
    }
  };

  if (tiles > 0) ld.load(0);
  if constexpr (NW > 1) {
    // two LDS buffers: behind the barrier tile t is whole in one and nobody reads the other, which tile t + 1 goes to
    unsigned groups = ld.groups;
    if (tiles > 0) {
      store_tile(0);
      if (tiles > 1) ld.load(1);
    }
    for (int t = 0; t < tiles; ++t) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      const unsigned now = groups;
      if (t + 1 < tiles) {
        groups = ld.groups;
        store_tile(t + 1);
        if (t + 2 < tiles) ld.load(t + 2);
      }
      work_tile(t, t & 1, now);
    }
  } else {
    // a wave's LDS operations are carried out in order: its own tile needs no barrier
    for (int t = 0; t < tiles; ++t) {
      const unsigned now = ld.groups;
      store_tile(t);
      if (t + 1 < tiles) ld.load(t + 1);
      work_tile(t, 0, now);
    }
  }
  float l_tot = l_run + __shfl_xor(l_run, 32, kWave);

  if constexpr (KW > 1) {
    // join the waves: waves 1 .. 3 leave (m, l, O), every wave sums a quarter of the channels in the waves' order
    __syncthreads();
    constexpr int OSTR = DHP + 4;                                  // floats per row: 16 bytes past the row against bank conflicts
    float *om = reinterpret_cast<float *>(smem);                   // [KW][32][OSTR] O, then [KW][32][2] m, l
    float *ml = om + KW * 32 * OSTR;
    static_assert(KW * 32 * (OSTR + 2) * 4 <= C::SMEM, "the partial results fit the tiles' LDS");
    float *mine = om + (wave * 32 + l32) * OSTR;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4 *>(mine + cb * 32 + 8 * g + 4 * hi) = make_float4(o[cb][4 * g], o[cb][4 * g + 1], o[cb][4 * g + 2], o[cb][4 * g + 3]);
    if (hi == 0) {
      ml[(wave * 32 + l32) * 2] = m_run;
      ml[(wave * 32 + l32) * 2 + 1] = l_tot;
    }
    __syncthreads();
    float m_all = -INFINITY;
#pragma unroll
    for (int v = 0; v < KW; ++v) m_all = fmaxf(m_all, ml[(v * 32 + l32) * 2]);
    const float m_use = m_all == -INFINITY ? 0.f : m_all;
    float wt[KW];
    l_tot = 0.f;
#pragma unroll
    for (int v = 0; v < KW; ++v) {
      wt[v] = __builtin_amdgcn_exp2f((ml[(v * 32 + l32) * 2] - m_use) * p.sl2);
      l_tot += wt[v] * ml[(v * 32 + l32) * 2 + 1];
    }
    m_run = m_all;
    // the lane's channels: 4 hi + 8 (wave + 4 i) .. + 3
    if (row.ok) {
      const float inv = l_tot != 0.f ? 1.f / l_tot : 0.f;
#pragma unroll
      for (int i = 0; i < (DHP / 8 + KW - 1) / KW; ++i) {
        const int c = 4 * hi + 8 * (wave + KW * i);
        if (c < dh) {
          float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int v = 0; v < KW; ++v) {
            const float4 x = *reinterpret_cast<const float4 *>(om + (v * 32 + l32) * OSTR + c);
            acc[0] = fmaf(wt[v], x.x, acc[0]);
            acc[1] = fmaf(wt[v], x.y, acc[1]);
            acc[2] = fmaf(wt[v], x.z, acc[2]);
            acc[3] = fmaf(wt[v], x.w, acc[3]);
          }
          put4<T>(a, w.sp, w.q0 + row.tok, row.head, c, inv, acc[0], acc[1], acc[2], acc[3]);
        }
      }
    }
  } else if (row.ok) {
    const float inv = l_tot != 0.f ? 1.f / l_tot : 0.f;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int c = cb * 32 + 8 * g + 4 * hi;
        if (c < dh) put4<T>(a, w.sp, w.q0 + row.tok, row.head, c, inv, o[cb][4 * g], o[cb][4 * g + 1], o[cb][4 * g + 2], o[cb][4 * g + 3]);
      }
  }
  if (row.ok && hi == 0 && (KW == 1 || wave == 0)) put_stats(a, w.sp, w.q0 + row.tok, row.head, m_run * p.sl2, l_tot);
  if (CAUSAL && w.zone < w.ke) {
    if constexpr (KW > 1) {
      // wave v's share of the keys, as above
      const int q = ((w.ke - w.kb + KW - 1) / KW + TK - 1) / TK * TK;
#pragma unroll 1
      for (int v = 0; v < KW; ++v) {
        const int b = min(w.ke, w.kb + v * q), e = min(w.ke, b + q);
        if (w.zone < e) add_hidden<T, PAGED, C::ROWS, 64 * C::WAVES>(p, w, hidden_all[v], ZONE * (TK / 32), b + (w.zone > b ? (w.zone - b) / TK : 0) * TK, e);
      }
    } else {
      __syncthreads();
      add_hidden<T, PAGED, C::ROWS, 64 * C::WAVES>(p, w, hidden, ZONE * (TK / 32), kb + zone_tile * TK, ke);
    }
  }
}

// The tile kernel for launches with many rows (bf16): four waves of 64 rows, one workgroup per CU.
//
// At 32 rows a wave every MFMA needs a 1 KB fragment from LDS: at the matrix units' rate that is all of the LDS's 128 bytes a
// clock.  With 64 rows two MFMAs share a fragment.  That leaves one wave per SIMD, so its vector work has to run under its own
// matrix work: a step on 32 keys is one block of instructions in which the score products of the next 32 keys and
// the value products of the 32 before go on while the vector unit turns the scores of this step into weights.
//
// Weights are taken relative to a reference exponent per row that is not the running maximum: p = 2^(s - ref) is right for
// any ref while nothing overflows, and the sum of a lane's weights, which is formed anyway, says when it has grown too
// large.  Only then (and on the first keys of a row, whose ref is -inf) is the maximum found, the reference moved, and the
// step's weights formed again.
template <int DHP, int KS, bool PAGED, bool CAUSAL>
__global__ __launch_bounds__(256, (DHP == 64 ? 2 : 1)) void attn_rows_wide_kernel(RowsKernelArgs p) {
  using T = bf16_t;
  using C = Tile<T, DHP, 4, 1>;
  constexpr int TK = C::TK, CB = C::CB;
  constexpr float kSumLimit = 8192.f;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];   // two K tiles, two V tiles
  unsigned char *const vring = smem + 2 * C::KTILE_B;
  const RowsAttn &a = p.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int l32 = lane & 31, hi = lane >> 5;
  const int dh = a.head_dim, G = p.group;
  Work w;
  if (!find_work<PAGED, CAUSAL, 256, 64>(p, lane, w)) return;
  if (empty_chunk<256>(p, w)) return;
  const int kb = __builtin_amdgcn_readfirstlane(w.kb), ke = __builtin_amdgcn_readfirstlane(w.ke);
  const int tiles = (ke - kb + TK - 1) / TK;

  // ---- the lane's two rows
  int limit[2];
  int least = ke;
  u32x4 qf[2][KS];
#pragma unroll
  for (int rb = 0; rb < 2; ++rb) {
    const LaneRow row(w, G, wave * 64 + rb * 32 + l32);
    limit[rb] = ke;
    if (CAUSAL && row.ok && w.first + row.tok + 1 < ke) limit[rb] = w.first + row.tok + 1 < 0 ? 0 : (int)(w.first + row.tok + 1);
    least = min(least, limit[rb]);
    const T *qp = (const T *)a.q + (int64_t)(w.q0 + row.tok) * a.ldq + (int64_t)row.head * dh;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      const int c = i * 16 + hi * 8;
      qf[rb][i] = u32x4{0, 0, 0, 0};
      if (row.ok && c < dh) qf[rb][i] = *reinterpret_cast<const u32x4 *>(qp + c);
    }
  }
  for (int o = 32; o > 0; o >>= 1) least = min(least, __shfl_xor(least, o, kWave));
  least = __builtin_amdgcn_readfirstlane(least);

  TileLoader<C, T, PAGED> ld(a, w, lane, wave, kb, ke);

  f32x16 o[2][CB];
#pragma unroll
  for (int rb = 0; rb < 2; ++rb)
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[rb][cb][i] = 0.f;
  float ref[2] = {-INFINITY, -INFINITY};     // reference exponents (of 2)
  float l_run[2] = {0.f, 0.f};

  const int i16 = lane & 15, g1 = (lane >> 4) & 1;
  const unsigned char *const k_at = smem + l32 * C::KROWB + hi * 16;
  const unsigned char *const v_at = vring + (4 * hi + (i16 >> 2)) * C::VROWB + g1 * 32 + (i16 & 3) * 8;

  struct Scores { f32x16 v[2]; };
  struct Weights { bf16x8 v[2][2]; };
  const f32x16 zero = {};
  constexpr int K_HALF = 32 * C::KROWB, V_HALF = 32 * C::VROWB;
  auto k_fragment = [&](int ks, int at) __attribute__((always_inline)) { return *reinterpret_cast<const bf16x8 *>(k_at + at + ks * 32); };
  auto v_fragment = [&](int j, int cb, int at) __attribute__((always_inline)) {
    struct { s16x4 lo, hi4; } v8 = {lds_read_transposed(v_at + at + j * 16 * C::VROWB + cb * 64), lds_read_transposed(v_at + at + (j * 16 + 8) * C::VROWB + cb * 64)};
    return __builtin_bit_cast(bf16x8, v8);
  };
  auto weights = [&](const f32x16 &x, float neg, bf16x8 (&y)[2]) __attribute__((always_inline)) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float e = __builtin_amdgcn_exp2f(fmaf(x[i], p.sl2, neg));
      sum += e;
      y[i >> 3][i & 7] = (bf16_t)e;
    }
    return sum;
  };
  // One step: weights of the 32 keys from key0 on (scores `cur`, pages `groups`), scores of the next 32 (K at kt), values of the 32
  // before (V at vt).  The registers of K (first half of a tile) or V (second) go to LDS at `side` and are loaded again.
  auto step = [&](int key0, unsigned groups, Scores &cur, Scores &nxt, const Weights &before, Weights &now, int kt, int vt, int side,
                  auto k_side) __attribute__((always_inline)) {
    if (key0 + 32 > least || (PAGED && groups != 3)) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = 8 * (i >> 2) + (i & 3);
          if (key0 + at + 4 * hi >= limit[rb] || (PAGED && !((groups >> (at >> 4)) & 1))) cur.v[rb][i] = -INFINITY;
        }
    }
    // The block, in slots of one MFMA with its share of the vector work behind it: an MFMA takes 32 cycles, in which the wave
    // can issue five other instructions.  Fragments come from LDS PD fragments ahead of their two MFMAs; an
    // element passes through its multiply-add, its exponential and its sum in slots behind each other.
    constexpr int NF = KS + 2 * CB, MF = 2 * NF, PD = 2;
    bf16x8 ring[PD + 1];
    auto fragment = [&](auto f_c) __attribute__((always_inline)) {
      constexpr int f = decltype(f_c)::value;
      if constexpr (f < KS) return k_fragment(f, kt);
      else return v_fragment((f - KS) / CB, (f - KS) % CB, vt);
    };
    unrolled<PD>([&](auto f_c) __attribute__((always_inline)) { ring[decltype(f_c)::value] = fragment(f_c); });
    float arg[32], e[32], sum[2] = {0.f, 0.f};
    unrolled<MF>([&](auto i_c) __attribute__((always_inline)) {
      constexpr int i = decltype(i_c)::value, f = i / 2, rb = i & 1;
      if constexpr (rb == 0 && f + PD < NF) ring[(f + PD) % (PD + 1)] = fragment(std::integral_constant<int, f + PD>{});
      const bf16x8 &fr = ring[f % (PD + 1)];
      if constexpr (f < KS) nxt.v[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr, __builtin_bit_cast(bf16x8, qf[rb][f]), f == 0 ? zero : nxt.v[rb], 0, 0, 0);
      else o[rb][(f - KS) % CB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr, before.v[rb][(f - KS) / CB], o[rb][(f - KS) % CB], 0, 0, 0);
      constexpr int u = i * C::LOADS / MF;
      if constexpr (i == 0 || u != (i - 1) * C::LOADS / MF) {
        if constexpr (decltype(k_side)::value) {
          ld.store_k(smem + side, u);
          ld.load_k(u);
        } else {
          ld.store_v(vring + side, u);
          ld.load_v(u);
        }
      }
      constexpr int N = MF - 2;
      auto from = [](int slot) { return slot < 0 ? 0 : slot > N ? 32 : slot * 32 / N; };
#pragma unroll
      for (int x = from(i); x < from(i + 1); ++x) {
        arg[x] = fmaf(cur.v[x >> 4][x & 15], p.sl2, -ref[x >> 4]);
        asm volatile("" : "+v"(arg[x]));   // stays in this slot
      }
#pragma unroll
      for (int x = from(i - 1); x < from(i); ++x) {
        e[x] = __builtin_amdgcn_exp2f(arg[x]);
        asm volatile("" : "+v"(e[x]));
      }
#pragma unroll
      for (int x = from(i - 2); x < from(i - 1); ++x) {
        sum[x >> 4] += e[x];
        if (x & 1) {
          const bf16x2 e2 = {(bf16_t)e[x - 1], (bf16_t)e[x]};
          unsigned u = __builtin_bit_cast(unsigned, e2);
          asm volatile("" : "+v"(u));      // rounded here, not behind the test of the sum where it is next used
          const bf16x2 r2 = __builtin_bit_cast(bf16x2, u);
          now.v[x >> 4][(x & 15) >> 3][(x & 7) - 1] = r2[0];
          now.v[x >> 4][(x & 15) >> 3][x & 7] = r2[1];
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    if (__builtin_amdgcn_ballot_w64(!(sum[0] < kSumLimit) || !(sum[1] < kSumLimit)) != 0) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) {
        float m = cur.v[rb][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) m = fmaxf(m, cur.v[rb][i]);
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
        m = fmaxf(ref[rb], fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * p.sl2);
        const float use = m == -INFINITY ? 0.f : m;                 // a row that has seen no key yet: weights 2^-inf = 0
        const float alpha = __builtin_amdgcn_exp2f(ref[rb] - use);
        ref[rb] = m;
        l_run[rb] *= alpha;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[rb][cb][i] *= alpha;
        sum[rb] = weights(cur.v[rb], -use, now.v[rb]);
      }
    }
    l_run[0] += sum[0];
    l_run[1] += sum[1];
  };

  // Tile t lies in LDS buffers t % 2.  Its first half's weights are formed while its second half's scores run, and so on.  K of tile t + 1
  // goes to LDS in the first half of tile t, where K of tile t - 1 has been read by all since the barrier before, V of tile t + 1 in
  // the second half, behind the barrier in the middle, from which on nobody reads V of tile t - 1.
  // keys with infinities or NaN among those that some row does not see (fewer than 256)
  constexpr int ZONE = 5;                                         // tiles they can touch
  __shared__ unsigned hidden[ZONE * 2];
  const bool zoned = CAUSAL && w.zone < ke;
  const int zone_tile = zoned && w.zone > kb ? (w.zone - kb) / TK : 0;
  if (zoned) {
    if (threadIdx.x < ZONE * 2) hidden[threadIdx.x] = 0;
    __syncthreads();
  }
  auto clear = [&](int t) __attribute__((always_inline)) {
    if (zoned && t >= zone_tile && t < tiles) ld.clear_v(hidden, t - zone_tile);
  };
  if (tiles > 0) {
    Scores s0, s1;
    Weights w0, w1;
#pragma unroll
    for (int rb = 0; rb < 2; ++rb)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) w1.v[rb][j][i] = (bf16_t)0.f;
    auto meet = [&]() __attribute__((always_inline)) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    };
    ld.load(0);
    unsigned groups_now = ld.groups;
    clear(0);
    ld.store(smem, vring);
    ld.load(1);
    unsigned groups_next = ld.groups;
    // the values "before tile 0" have weight zero, so that they must be finite: the other V buffer's second half
    static_assert(V_HALF % 1024 == 0, "whole kilobytes, one a wave and turn");
    for (int i = wave; i < V_HALF / 1024; i += 4) *reinterpret_cast<u32x4 *>(vring + C::VTILE_B + V_HALF + i * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
    meet();
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 kf = k_fragment(ks, 0);
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) s0.v[rb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, __builtin_bit_cast(bf16x8, qf[rb][ks]), ks == 0 ? zero : s0.v[rb], 0, 0, 0);
    }
    auto last_values = [&](int at) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          const bf16x8 vf = v_fragment(j, cb, at);
#pragma unroll
          for (int rb = 0; rb < 2; ++rb) o[rb][cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, w1.v[rb][j], o[rb][cb], 0, 0, 0);
        }
    };
    for (int t = 0; t < tiles; ++t) {
      const int key0 = kb + t * TK;
      const int k0 = t & 1 ? C::KTILE_B : 0, k1 = C::KTILE_B - k0, v0 = t & 1 ? C::VTILE_B : 0, v1 = C::VTILE_B - v0;
      ld.aim(t + 2);
      step(key0, groups_now & 3, s0, s1, w1, w0, k0 + K_HALF, v1 + V_HALF, k1, std::true_type{});
      meet();
      clear(t + 1);
      step(key0 + 32, groups_now >> 2, s1, s0, w0, w1, k1, v0, v1, std::false_type{});
      groups_now = groups_next;
      groups_next = ld.groups;
    }
    last_values((tiles & 1 ? 0 : C::VTILE_B) + V_HALF);
  }

  int lane_again = l32;                          // the rows are worked out anew here, not kept in registers through the loop
  asm volatile("" : "+v"(lane_again));
#pragma unroll
  for (int rb = 0; rb < 2; ++rb) {
    const float l = l_run[rb] + __shfl_xor(l_run[rb], 32, kWave);
    const LaneRow row(w, G, wave * 64 + rb * 32 + lane_again);
    if (!row.ok) continue;
    const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int c = cb * 32 + 8 * g + 4 * hi;
        if (c < dh) put4<T>(a, w.sp, w.q0 + row.tok, row.head, c, inv, o[rb][cb][4 * g], o[rb][cb][4 * g + 1], o[rb][cb][4 * g + 2], o[rb][cb][4 * g + 3]);
      }
    if (hi == 0) put_stats(a, w.sp, w.q0 + row.tok, row.head, ref[rb], l);
  }
  if (zoned) {
    __syncthreads();
    add_hidden<T, PAGED, 256, 256>(p, w, hidden, ZONE * 2, kb + zone_tile * TK, ke);
  }
}

// Joins the chunks of a row: out = sum 2^(m_c - m) O_c / sum 2^(m_c - m) l_c, W waves per (token, head).  A thread sums four channels of
// every GROUPS-th chunk, the groups are added up through LDS in their order.  Chunks that saw no key of the row left l = 0; their O is
// not used.  One whose weight is 0 only in 32 bits is: its infinities and NaN reach the row, as they do where the keys are one chunk.  Four to five microseconds, launch included, of three memory latencies behind each other, for a token of 16 heads in 128
// chunks as for 64 of 32 heads in 8.
template <typename T, int W>
__global__ __launch_bounds__(256) void attn_rows_join_kernel(RowsAttn a) {
  constexpr int R = 4 / W, NT = 64 * W;                       // rows per workgroup, threads per row
  __shared__ float weight[R][kMaxChunks], part[R][NT * 4], stat[R][2 * W];
  const int slot = threadIdx.x / NT, tid = threadIdx.x % NT, lane = threadIdx.x & 63, wave = tid >> 6;
  const int dh = a.head_dim;
  const int64_t all = (int64_t)a.total_q * a.n_heads;
  const int64_t id = (int64_t)blockIdx.x * R + slot;
  const int row = (int)(min(id, all - 1) / a.n_heads), head = (int)(min(id, all - 1) - (int64_t)row * a.n_heads);
  const bool live = id < all && row >= a.cu_q[0] && row < a.cu_q[a.n_seqs];
  const float2 *ml = reinterpret_cast<const float2 *>(a.ws + (int64_t)a.splits * all * dh) + id;
  constexpr int PER = (kMaxChunks + NT - 1) / NT;
  constexpr float kNone = -1.f;                               // in place of a weight: no key
  float2 v[PER];
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    v[i] = make_float2(-INFINITY, 0.f);
    if (live && i * NT + tid < a.splits) v[i] = ml[(i * NT + tid) * all];
    m = fmaxf(m, v[i].x);
  }
  m = wave_max(m);
  if (lane == 0) stat[slot][wave] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < W; ++i) m = fmaxf(m, stat[slot][i]);
  float l = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i)
    if (i * NT + tid < a.splits) {
      const float w = v[i].y != 0.f ? __builtin_amdgcn_exp2f(v[i].x - m) : kNone;
      weight[slot][i * NT + tid] = w;
      if (w != kNone) l = fmaf(w, v[i].y, l);
    }
  l = wave_sum(l);
  if (lane == 0) stat[slot][W + wave] = l;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int i = 0; i < W; ++i) l += stat[slot][W + i];
  const int cl = dh <= 64 ? 16 : 32, groups = NT / cl;        // threads across a row's channels
  const int c = tid % cl * 4, g = tid / cl;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  if (live && c < dh) {
    // eight chunks' loads at a time, whether they count or not (a chunk that does not may hold anything)
    for (int i0 = g; i0 < a.splits; i0 += 8 * groups) {
      float4 x[8];
      float w[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int i = min(i0 + j * groups, a.splits - 1);
        x[j] = *reinterpret_cast<const float4 *>(a.ws + ((int64_t)i * all + id) * dh + c);
        w[j] = i0 + j * groups < a.splits ? weight[slot][i] : kNone;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (w[j] != kNone) acc = make_float4(fmaf(w[j], x[j].x, acc.x), fmaf(w[j], x[j].y, acc.y), fmaf(w[j], x[j].z, acc.z), fmaf(w[j], x[j].w, acc.w));
    }
  }
  *reinterpret_cast<float4 *>(&part[slot][tid * 4]) = acc;
  __syncthreads();
  if (!live) return;
  const float inv = l != 0.f ? 1.f / l : 0.f;
  if (g == 0 && c < dh) {
    for (int i = 1; i < groups; ++i) {
      const float4 x = *reinterpret_cast<const float4 *>(&part[slot][(i * cl + tid) * 4]);
      acc = make_float4(acc.x + x.x, acc.y + x.y, acc.z + x.z, acc.w + x.w);
    }
    T *dst = (T *)a.out + (int64_t)row * a.ldo + (int64_t)head * dh + c;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(dst) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    else *reinterpret_cast<bf16x4 *>(dst) = bf16x4{(bf16_t)(acc.x * inv), (bf16_t)(acc.y * inv), (bf16_t)(acc.z * inv), (bf16_t)(acc.w * inv)};
  }
  if (a.lse && tid == 0) a.lse[id] = l != 0.f ? m * kLn2 + logf(l) : -INFINITY;
}

template <typename T>
hipError_t launch_join(const RowsAttn &a, hipStream_t s) {
  const int64_t all = (int64_t)a.total_q * a.n_heads;
  // four waves per row where a wave would have more than eight chunks to add up per thread (128 chunks of a token of 16 heads: the call
  // takes 30.9 us, with one wave 34.4; 16 chunks of 64 tokens of 32 heads: 176, with four waves 180)
  if (a.splits > 16) attn_rows_join_kernel<T, 4><<<dim3((unsigned)all), 256, 0, s>>>(a);
  else attn_rows_join_kernel<T, 1><<<dim3((unsigned)((all + 3) / 4)), 256, 0, s>>>(a);
  return hipGetLastError();
}

// Workgroups of `per` rows that have rows, without chunks.
int64_t workgroups(int64_t total_q, int group, int n_seqs, int kv_heads, int per) {
  return std::max((total_q * group + per - 1) / per, (int64_t)n_seqs) * kv_heads;
}
// Two workgroups of head size 64, or of the key kernel, fit a CU, and the dispatcher puts them there while other CUs are idle: where
// there are no more than CUs, each asks for more than half a CU's LDS (4 x 512 rows x 24 heads over 4250 keys 132 -> 95 us; 8 tokens of
// 8 key heads over 4096 keys in four chunks 37.6 -> 30.4).
constexpr int kAloneBytes = 82 * 1024;
bool few_workgroups(const RowsAttn &a, int per) {
  return workgroups(a.total_q, a.n_heads / a.kv_heads, a.n_seqs, a.kv_heads, per) * a.splits <= 256;
}

template <typename T, int DHP, bool PAGED, bool CAUSAL, int NW, int KW>
hipError_t launch_shape(const RowsAttn &a, hipStream_t s) {
  using C = Tile<T, DHP, NW, KW>;
  constexpr int alone = KW > 1 && C::SMEM < kAloneBytes ? kAloneBytes : C::SMEM;
  if (hipError_t e = allow_dynamic_lds<&attn_rows_kernel<T, DHP, PAGED, CAUSAL, NW, KW>, alone>(); e != hipSuccess) return e;
  RowsKernelArgs p{a, a.n_heads / a.kv_heads, 0, a.scale * kLog2e};
  p.slots = (int)((int64_t)a.total_q * p.group / C::ROWS) + a.n_seqs;
  const int64_t grid = (int64_t)p.slots * a.splits * a.kv_heads;
  attn_rows_kernel<T, DHP, PAGED, CAUSAL, NW, KW><<<dim3((unsigned)grid), 64 * C::WAVES, few_workgroups(a, C::ROWS) ? alone : C::SMEM, s>>>(p);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || a.splits == 1 ? e : launch_join<T>(a, s);
}

template <int DHP, int KS, bool PAGED, bool CAUSAL>
hipError_t launch_wide(const RowsAttn &a, hipStream_t s) {
  constexpr int smem = Tile<bf16_t, DHP, 4, 1>::SMEM, alone = smem > kAloneBytes ? smem : kAloneBytes;
  if (hipError_t e = allow_dynamic_lds<&attn_rows_wide_kernel<DHP, KS, PAGED, CAUSAL>, alone>(); e != hipSuccess) return e;
  RowsKernelArgs p{a, a.n_heads / a.kv_heads, 0, a.scale * kLog2e};
  p.slots = (int)((int64_t)a.total_q * p.group / 256) + a.n_seqs;
  const int64_t grid = (int64_t)p.slots * a.splits * a.kv_heads;
  attn_rows_wide_kernel<DHP, KS, PAGED, CAUSAL><<<dim3((unsigned)grid), 256, few_workgroups(a, 256) ? alone : smem, s>>>(p);
  const hipError_t e = hipGetLastError();
  return e != hipSuccess || a.splits == 1 ? e : launch_join<bf16_t>(a, s);
}

template <typename T, int DHP, bool PAGED, bool CAUSAL>
hipError_t launch_rows_of(const RowsAttn &a, hipStream_t s) {
  if (a.shape == ROWS_KEYS) return launch_shape<T, DHP, PAGED, CAUSAL, 1, 4>(a, s);
  if constexpr (sizeof(T) == 2) {
    if (a.shape == ROWS_WIDE) {
      // head sizes up to 80: five steps of 16 channels for the scores, of the six that a row of 96 has
      if constexpr (DHP == 96) {
        if (a.head_dim <= 80) return launch_wide<DHP, 5, PAGED, CAUSAL>(a, s);
      }
      return launch_wide<DHP, DHP / 16, PAGED, CAUSAL>(a, s);
    }
  }
  return launch_shape<T, DHP, PAGED, CAUSAL, 4, 1>(a, s);
}
template <typename T, bool PAGED, bool CAUSAL>
hipError_t launch_dim(const RowsAttn &a, hipStream_t s) {
  if (a.head_dim <= 64) return launch_rows_of<T, 64, PAGED, CAUSAL>(a, s);
  if (a.head_dim <= 96) return launch_rows_of<T, 96, PAGED, CAUSAL>(a, s);
  return launch_rows_of<T, 128, PAGED, CAUSAL>(a, s);
}
template <typename T>
hipError_t launch_type(const RowsAttn &a, hipStream_t s) {
  if (a.pages.table) return a.causal ? launch_dim<T, true, true>(a, s) : launch_dim<T, true, false>(a, s);
  return a.causal ? launch_dim<T, false, true>(a, s) : launch_dim<T, false, false>(a, s);
}

}  // namespace

// Which kernel, and how many chunks of the key range, by the estimated time in microseconds.  The lengths are on the device: the host
// knows the rows of all sequences, their number, and that none has more than max_kv keys; a causal mask and shorter
// sequences make all the estimates too long alike.
RowsPlan rows_attention_plan(int dt, int total_q, int n_seqs, int n_heads, int kv_heads, int head_dim, int64_t max_kv) {
  const int64_t rows = (int64_t)total_q * (n_heads / kv_heads), tiles = (max_kv + 63) / 64;
  const auto wgs = [&](int per) { return workgroups(total_q, n_heads / kv_heads, n_seqs, kv_heads, per); };
  const auto rounds = [](int64_t n, int fit) { return n <= 2 * fit ? (double)((n + fit - 1) / fit) : (double)n / fit + 0.5; };
  // the second launch, and the partial results on their way through memory (4 TB/s)
  const double row_us = (double)total_q * n_heads * head_dim * 4.9e-7;
  const auto join_us = [&](int64_t n) { return n > 1 ? 4.0 + (4 * n + 2) * row_us : 0.0; };
  const int dim = head_dim <= 64 ? 0 : head_dim <= 96 ? 1 : 2;

  RowsPlan p{ROWS_TILES, 1, 0, 0};
  double best = 1e300;
  const auto offer = [&](int shape, int64_t n, double us) {
    if (us < best - 1e-9) {
      best = us;
      p = RowsPlan{shape, (int)n, 256, 0};
    }
  };
  // chunks of four tiles or more, and none for launches that fill the chip twice without
  const int64_t most = tiles < 8 ? 1 : tiles / 4 < 16 ? tiles / 4 : 16;
  for (int64_t n = 1; n <= most; ++n) {
    const double steps = (double)((tiles + n - 1) / n);
    // 128 rows: two workgroups fit a CU; a tile of 64 keys takes this long where a CU has one, and where it has two (head sizes 64, 96, 128)
    constexpr double kOne[] = {0.9, 1.4, 1.5}, kTwo[] = {1.3, 1.9, 2.3};
    const int64_t w = wgs(128) * n;
    if (w - wgs(128) < 1024) offer(ROWS_TILES, n, rounds(w, 512) * (steps + 4) * (w <= 256 ? kOne[dim] : kTwo[dim]) + join_us(n));
    // 256 rows, one on a CU (2048 rows x 16 heads of 72 over 2048 keys: 44 us against 59)
    constexpr double kWide[] = {1.0, 1.2, 1.7};
    if (dt == DT_BF16 && wgs(256) * (n - 1) < 512) offer(ROWS_WIDE, n, rounds(wgs(256) * n, 256) * (steps * kWide[dim] + 8) + join_us(n));
  }

  // The key kernel for single tokens, and for launches that leave the chip empty.  It reads the keys for every 32 rows, through the
  // L2s at some 8 TB/s (1024 rows x 16 heads of 72 over 1024 keys: 18 us, in tiles 30; 512 rows x 8 heads of 128 over 16384
  // keys: 188 and 63).  In fp32 the matrix units bound all kernels, and more waves are better until the chip holds them (1024
  // rows x 16 heads of 128 over as many keys: 88 us, in tiles 121).
  const double keys_us = 4.0 + (double)wgs(32) * max_kv * head_dim * 2 * dt_size(dt) / 8e6;
  if (rows <= (int64_t)n_seqs * 32 || (dt == DT_BF16 ? keys_us < best : wgs(32) <= 1024)) {
    // Chunks down to 256 keys while there is no more than a workgroup for every CU (one token of 8 key heads over 4096 keys: 16 chunks
    // 13.5 us, 4 chunks 21.3; of 2 key heads over 131072 keys: 128 chunks 30.6 us, 64 chunks 34.0, 256 chunks 33.0; 20 tokens of 8
    // over 4096: whole 54, in two chunks 66).  Behind that, chunks of at least 2048 keys, whole rounds of the 512
    // workgroups that the chip holds, up to 8192: caches of different lengths share the chip evenly (64 tokens over up to 16384 keys of
    // 8 key heads: 150 us, without chunks 211, with chunks of 1024 keys 177; where lengths are alike it costs little: 32 tokens
    // over 8192 keys each 176, in two chunks 173).
    const int64_t w = wgs(32), none = 1;
    int64_t n = std::min(std::max(256 / w, none), std::max(max_kv / 256, none));
    int64_t more = std::min((8192 + w - 1) / w, max_kv / 2048);
    if (w < 512) more -= more % (512 / w);
    n = std::max(n, more);
    p = RowsPlan{ROWS_KEYS, (int)(n < kMaxChunks ? n : kMaxChunks), n == more ? 2048 : 256, 0};
  }
  if (p.splits > 1) p.ws_bytes = (size_t)p.splits * total_q * n_heads * (head_dim + 2) * sizeof(float);
  return p;
}

hipError_t launch_rows_attention(const RowsAttn &a, hipStream_t s) {
  return a.dt == DT_BF16 ? launch_type<bf16_t>(a, s) : launch_type<float>(a, s);
}

}  // namespace pf
