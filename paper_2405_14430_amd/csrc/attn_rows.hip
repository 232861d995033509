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
// The keys of a launch with few workgroups are cut into chunks, whose partial results a second launch joins.
//
// Tiles come from memory through registers: while the products of tile t run, the loads of tile t + 1 are in flight.  The
// bounds of the buffer loads give zeros for rows past the last key, for pages that are none and for channels past the head, so
// neither the scores nor 0 * v meets what lies there.  LDS rows are swizzled by 16-byte pieces against bank conflicts.
#include "requests.h"

namespace pf {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

#if defined(__HIP_DEVICE_COMPILE__)
struct Buffer {   // `bytes` bytes from a wave-uniform address; loads past them give zeros
  __amdgpu_buffer_rsrc_t rs;
  __device__ __forceinline__ Buffer(const void *base, unsigned bytes)
      : rs(__builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, bytes, 0x00020000)) {}
  __device__ __forceinline__ u32x4 load16(unsigned at) const {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, at, 0, 0));
  }
};
__device__ __forceinline__ s16x4 lds_read_transposed(const unsigned char *p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p);
}
#else   // the host pass only parses the kernels
struct Buffer {
  __device__ Buffer(const void *, unsigned) {}
  __device__ u32x4 load16(unsigned) const { return u32x4{}; }
};
__device__ s16x4 lds_read_transposed(const unsigned char *) { return s16x4{}; }
#endif

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
  static constexpr int CHUNKS = ROWB / 16;
  static constexpr int TILE_B = TK * ROWB;
  static constexpr int RW = TK / NW;                       // rows of a tile that one wave brings in
  static constexpr int LOADS = RW * ROWB / 1024;           // its 1 KB loads
  static constexpr int BUFS = NW > 1 ? 2 : 1;
  static constexpr int JOIN_B = KW > 1 ? KW * 32 * (DHP + 4 + 2) * 4 : 0;   // the waves' partial results
  static constexpr int SMEM = KW * BUFS * 2 * TILE_B > JOIN_B ? KW * BUFS * 2 * TILE_B : JOIN_B;
  static constexpr int ROWS = 32 * NW;                     // query rows of a workgroup
  static constexpr int WGS = SMEM > 80 * 1024 ? 1 : 2;     // workgroups on a CU, by their LDS
  // swizzles of the 16-byte pieces of LDS row r: K is read as 16 bytes of 16 rows at a time, V as 64 bytes of four rows
  // (transposed, bf16) or 128 bytes of rows r and r + 4 (fp32)
  static __device__ __forceinline__ constexpr int kkey(int r) {
    return ROWB % 256 == 0 ? (r & 15) : ROWB == 128 ? ((r >> 1) & 7) : ROWB == 192 ? ((r >> 2) & 3) : ((r >> 1) & 7);
  }
  static __device__ __forceinline__ constexpr int vkey(int r) {
    return F32 ? (ROWB % 256 == 0 ? ((r >> 2) & 1) << 3 : 0) : ROWB == 256 ? (r & 3) << 2 : ROWB == 128 ? ((r >> 1) & 1) << 2 : 0;
  }
};

// Key tiles of one chunk when the longest sequence of the launch is cut into `splits` of them: at least four.
__device__ __forceinline__ int chunk_tiles(int longest_tiles, int splits) {
  const int c = (longest_tiles + splits - 1) / splits;
  return c < 4 ? 4 : c;
}
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

template <typename T, int DHP, bool PAGED, int NW, int KW>
__global__ __launch_bounds__(64 * NW * KW, (Tile<T, DHP, NW, KW>::WGS)) void attn_rows_kernel(RowsKernelArgs p) {
  using C = Tile<T, DHP, NW, KW>;
  constexpr int TK = C::TK, NB = C::NB, CB = C::CB, ROWB = C::ROWB;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const RowsAttn &a = p.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int l32 = lane & 31, hi = lane >> 5;
  const int dh = a.head_dim, G = p.group;

  // ---- workgroup -> (key head, row tile, chunk).  Neighbouring ids are different key heads: ids go round the 8 XCDs, so with 8
  // or more key heads a head's workgroups meet in one L2.  Later row tiles, which see more keys, come first.
  const int hk = blockIdx.x % a.kv_heads, rest = blockIdx.x / a.kv_heads;
  const int sp = rest % a.splits, slot = p.slots - 1 - rest / a.splits;
  // row tiles of sequence s: slots floor(cu[s] G / ROWS) + s and on, enough for any start of the sequence
  const int s = wave_search(a.n_seqs - 1, lane, slot, [&](int i) { return clampi(a.cu_q[i], 0, a.total_q) * G / C::ROWS + i; });
  if (s < 0) return;
  int q0, q1;
  sequence_rows(a.cu_q, s, a.total_q, q0, q1);
  const int n = q1 - q0;
  const int r_first = (slot - (q0 * G / C::ROWS + s)) * C::ROWS;
  if (r_first < 0 || r_first >= n * G) return;

  // ---- keys: those of the sequence, for causal rows up to the tile's last row's; the chunk's share of them
  int k0;
  const int kn = sequence_keys<PAGED>(a, s, k0);
  const int64_t first = !a.causal ? 0 : PAGED ? a.first[s] : kn - n;      // the slot of query 0
  const int t_last = (r_first + C::ROWS < n * G ? r_first + C::ROWS - 1 : n * G - 1) / G;
  int k_end = kn;
  if (a.causal && first + t_last + 1 < k_end) k_end = first + t_last + 1 < 0 ? 0 : (int)(first + t_last + 1);
  constexpr int UNIT = 64 * KW;      // keys per chunk tile: a multiple of what all waves walk in a step
  int kb = 0, ke = k_end;
  if (a.splits > 1) {
    int longest = 0;
    for (int i = lane; i < a.n_seqs; i += 64) {
      int unused;
      longest = max(longest, sequence_keys<PAGED>(a, i, unused));
    }
    for (int o = 32; o > 0; o >>= 1) longest = max(longest, __shfl_xor(longest, o, kWave));
    const int64_t c = (int64_t)chunk_tiles((longest + UNIT - 1) / UNIT, a.splits) * UNIT;
    kb = (int)min((int64_t)k_end, sp * c);
    ke = (int)min((int64_t)k_end, (sp + 1) * c);
  }
  if constexpr (KW > 1) {            // the wave's quarter
    const int q = ((ke - kb + KW - 1) / KW + TK - 1) / TK * TK;
    const int wb = min(ke, kb + (wave / NW) * q);
    ke = min(ke, wb + q);
    kb = wb;
  }
  kb = __builtin_amdgcn_readfirstlane(kb);
  ke = __builtin_amdgcn_readfirstlane(ke);
  const int tiles = (ke - kb + TK - 1) / TK;

  // ---- the lane's row
  const int wr = KW > 1 ? 0 : wave;
  const int r = r_first + wr * 32 + l32;
  const bool row_ok = r < n * G;
  const int tok = row_ok ? r / G : 0;
  const int head = hk * G + (row_ok ? r - tok * G : 0);
  int limit = ke;                    // keys before this one are seen
  if (row_ok && a.causal && first + tok + 1 < limit) limit = first + tok + 1 < 0 ? 0 : (int)(first + tok + 1);
  int least = limit;                 // of all rows of the wave: tiles below it need no mask
  for (int o = 32; o > 0; o >>= 1) least = min(least, __shfl_xor(least, o, kWave));
  least = __builtin_amdgcn_readfirstlane(least);

  // ---- Q fragments: bf16: channels ks * 16 + 8 hi .. + 7; fp32: channels j * 8 + 4 hi .. + 3
  constexpr int NQ = C::F32 ? DHP / 8 : DHP / 16;
  u32x4 qf[NQ];
  {
    const T *qp = (const T *)a.q + (int64_t)(q0 + tok) * a.ldq + (int64_t)head * dh;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
      const int c = C::F32 ? i * 8 + hi * 4 : i * 16 + hi * 8;
      qf[i] = u32x4{0, 0, 0, 0};
      if (row_ok && c < dh) qf[i] = *reinterpret_cast<const u32x4 *>(qp + c);
    }
  }

  // ---- tile loads.  A wave brings in rows [w * RW, (w + 1) * RW) of a tile, all of one 16-row group, so of one page (the key
  // kernel's 32 rows: two groups, loaded one after the other).
  const int lw = KW > 1 ? 0 : wave;
  constexpr int GROUPS = C::RW > 16 ? C::RW / 16 : 1;            // page groups a wave loads per tile
  constexpr int GL = C::LOADS / GROUPS;                           // loads per group
  constexpr int GROWS = C::RW / GROUPS;
  const unsigned k_row = (unsigned)((PAGED ? (int64_t)dh : a.ldk) * (int64_t)sizeof(T));
  const unsigned v_row = (unsigned)((PAGED ? (int64_t)dh : a.ldv) * (int64_t)sizeof(T));
  constexpr unsigned kOutside = 0x7fff0000u;
  unsigned k_off[C::LOADS], v_off[C::LOADS];                      // from the group's first row
#pragma unroll
  for (int i = 0; i < C::LOADS; ++i) {
    const int off = i * 1024 + lane * 16, row = off / ROWB, piece = (off % ROWB) >> 4;
    const int in_tile = lw * C::RW + row, in_group = row % GROWS;
    const int kc = piece ^ C::kkey(in_tile), vc = piece ^ C::vkey(in_tile);
    k_off[i] = kc * 16 < dh * (int)sizeof(T) ? in_group * k_row + kc * 16 : kOutside;
    v_off[i] = vc * 16 < dh * (int)sizeof(T) ? in_group * v_row + vc * 16 : kOutside;
  }
  unsigned char *const ring = smem + (KW > 1 ? (wave / NW) * C::BUFS * 2 * C::TILE_B : 0);
  const T *const k_head = PAGED ? (const T *)a.pages.k + ((int64_t)hk << a.pages.page_shift) * dh : (const T *)a.k + (int64_t)k0 * a.ldk + (int64_t)hk * dh;
  const T *const v_head = PAGED ? (const T *)a.pages.v + ((int64_t)hk << a.pages.page_shift) * dh : (const T *)a.v + (int64_t)k0 * a.ldv + (int64_t)hk * dh;

  // Pages: lane i holds the page of 16-key group i of the current 1024 keys, and of the next 1024 (loaded that far ahead).
  // kb is a multiple of TK; groups count from kb rounded down to 16.
  constexpr int TPB = 1024 / TK;                                  // tiles per block of 64 groups
  int page_now = -1, page_next = -1;
  auto table_entry = [&](int block) __attribute__((always_inline)) {
    const int64_t key = (int64_t)kb + block * 1024 + lane * 16;
    int pg = -1;
    if (key < ke) pg = a.pages.table[(int64_t)s * a.pages.max_pages + (key >> a.pages.page_shift)];
    return pg >= 0 && pg < a.pages.n_pages ? pg : -1;
  };
  if constexpr (PAGED) page_next = table_entry(0);

  u32x4 k_reg[C::LOADS], v_reg[C::LOADS];
  unsigned groups_ahead = 0;        // which 16-key groups of the tile in the registers have a page
  auto load_tile = [&](int t) __attribute__((always_inline)) {
    if constexpr (PAGED) {
      if (t % TPB == 0) {
        page_now = page_next;
        page_next = table_entry(t / TPB + 1);
      }
      groups_ahead = (unsigned)(__builtin_amdgcn_ballot_w64(page_now >= 0) >> ((t % TPB) * (TK / 16))) & ((1u << (TK / 16)) - 1);
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const int key = kb + t * TK + lw * C::RW + g * GROWS;       // wave-uniform
      int rows = clampi(ke - key, 0, GROWS);
      const T *ks, *vs;
      if constexpr (PAGED) {
        const int pg = __builtin_amdgcn_readlane(page_now, (t % TPB) * (TK / 16) + ((lw * C::RW + g * GROWS) >> 4));
        if (pg < 0) rows = 0;
        const int64_t at = (int64_t)(key & ((1 << a.pages.page_shift) - 1)) * dh;
        ks = k_head + (pg < 0 ? 0 : pg * a.pages.k_stride + at);
        vs = v_head + (pg < 0 ? 0 : pg * a.pages.v_stride + at);
      } else {
        ks = k_head + (rows ? key * a.ldk : 0);
        vs = v_head + (rows ? key * a.ldv : 0);
      }
      const Buffer kbuf(ks, rows * k_row), vbuf(vs, rows * v_row);
#pragma unroll
      for (int i = 0; i < GL; ++i) k_reg[g * GL + i] = kbuf.load16(k_off[g * GL + i]);
#pragma unroll
      for (int i = 0; i < GL; ++i) v_reg[g * GL + i] = vbuf.load16(v_off[g * GL + i]);
    }
  };
  auto store_tile = [&](int buf) __attribute__((always_inline)) {
    unsigned char *kd = ring + buf * 2 * C::TILE_B + lw * C::RW * ROWB + lane * 16, *vd = kd + C::TILE_B;
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) *reinterpret_cast<u32x4 *>(kd + i * 1024) = k_reg[i];
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) *reinterpret_cast<u32x4 *>(vd + i * 1024) = v_reg[i];
  };

  f32x16 o[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[cb][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;    // running maximum of the raw scores; the lane's share of the sum

  // LDS addresses of the lane: K row l32; V, bf16: row 4 hi + (i >> 2), piece of channels 16 g1 + 4 (i & 3); fp32: row 4 hi, channel l32
  const int i16 = lane & 15, g1 = (lane >> 4) & 1;
  const int v_row0 = C::F32 ? 4 * hi : 4 * hi + (i16 >> 2);
  int v_at[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) {
    const int piece = C::F32 ? cb * 8 + (l32 >> 2) : cb * 4 + g1 * 2 + ((i16 & 3) >> 1);
    v_at[cb] = v_row0 * ROWB + ((piece ^ C::vkey(v_row0)) << 4) + (C::F32 ? (l32 & 3) * 4 : (i16 & 1) * 8);
  }

  auto work_tile = [&](int t, int buf, unsigned groups) __attribute__((always_inline)) {
    const unsigned char *kt = ring + buf * 2 * C::TILE_B, *vt = kt + C::TILE_B;
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
          const bf16x8 kf = *reinterpret_cast<const bf16x8 *>(kt + (b * 32 + l32) * ROWB + (((ks * 2 + hi) ^ C::kkey(l32)) << 4));
          sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, __builtin_bit_cast(bf16x8, qf[ks]), sc[b], 0, 0, 0);
        }
    } else {
#pragma unroll
      for (int j = 0; j < DHP / 8; ++j) {
        const f32x4 kf = *reinterpret_cast<const f32x4 *>(kt + l32 * ROWB + (((j * 2 + hi) ^ C::kkey(l32)) << 4));
        const f32x4 qv = __builtin_bit_cast(f32x4, qf[j]);
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[e], qv[e], sc[0], 0, 0, 0);
      }
    }
    const int key0 = kb + t * TK;
    if (key0 + TK > least || (PAGED && groups != (1u << (TK / 16)) - 1)) {
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
          struct { s16x4 lo, hi4; } v8 = {lds_read_transposed(vt + v_at[cb] + j * 16 * ROWB), lds_read_transposed(vt + v_at[cb] + (j * 16 + 8) * ROWB)};
          o[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, v8), pf, o[cb], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          // the swizzle looks at bit 2 of the row, which 4 hi alone sets: rows 8 (i / 4) + i % 4 only move by whole rows
          const float vf = *reinterpret_cast<const float *>(vt + v_at[cb] + (8 * (i >> 2) + (i & 3)) * ROWB);
          o[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, sc[0][i], o[cb], 0, 0, 0);
        }
    }
  };

  if (tiles > 0) load_tile(0);
  if constexpr (NW > 1) {
    // two LDS buffers: behind the barrier tile t is whole in one and nobody reads the other, which tile t + 1 goes to
    unsigned groups = groups_ahead;
    if (tiles > 0) {
      store_tile(0);
      if (tiles > 1) load_tile(1);
    }
    for (int t = 0; t < tiles; ++t) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      const unsigned now = groups;
      if (t + 1 < tiles) {
        groups = groups_ahead;
        store_tile((t + 1) & 1);
        if (t + 2 < tiles) load_tile(t + 2);
      }
      work_tile(t, t & 1, now);
    }
  } else {
    // a wave's LDS operations are carried out in order: its own tile needs no barrier
    for (int t = 0; t < tiles; ++t) {
      const unsigned now = groups_ahead;
      store_tile(0);
      if (t + 1 < tiles) load_tile(t + 1);
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
    for (int w = 0; w < KW; ++w) m_all = fmaxf(m_all, ml[(w * 32 + l32) * 2]);
    const float m_use = m_all == -INFINITY ? 0.f : m_all;
    float wt[KW];
    l_tot = 0.f;
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      wt[w] = __builtin_amdgcn_exp2f((ml[(w * 32 + l32) * 2] - m_use) * p.sl2);
      l_tot += wt[w] * ml[(w * 32 + l32) * 2 + 1];
    }
    m_run = m_all;
    // the lane's channels: 4 hi + 8 (wave + 4 i) .. + 3
    if (row_ok) {
      const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
      const int64_t qr = q0 + tok;
#pragma unroll
      for (int i = 0; i < (DHP / 8 + KW - 1) / KW; ++i) {
        const int c = 4 * hi + 8 * (wave + KW * i);
        if (c < dh) {
          float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int w = 0; w < KW; ++w) {
            const float4 x = *reinterpret_cast<const float4 *>(om + (w * 32 + l32) * OSTR + c);
            acc[0] = fmaf(wt[w], x.x, acc[0]);
            acc[1] = fmaf(wt[w], x.y, acc[1]);
            acc[2] = fmaf(wt[w], x.z, acc[2]);
            acc[3] = fmaf(wt[w], x.w, acc[3]);
          }
          if (a.splits > 1) {
            float *dst = a.ws + (((int64_t)sp * a.total_q + qr) * a.n_heads + head) * dh + c;
            *reinterpret_cast<float4 *>(dst) = make_float4(acc[0], acc[1], acc[2], acc[3]);
          } else {
            T *dst = (T *)a.out + qr * a.ldo + (int64_t)head * dh + c;
            if constexpr (C::F32) {
              *reinterpret_cast<float4 *>(dst) = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
            } else {
              bf16x4 v;
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] = (bf16_t)(acc[e] * inv);
              *reinterpret_cast<bf16x4 *>(dst) = v;
            }
          }
        }
      }
    }
    if (wave != 0) return;
  } else if (row_ok) {
    const float inv = l_tot > 0.f ? 1.f / l_tot : 0.f;
    const int64_t qr = q0 + tok;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int c = cb * 32 + 8 * g + 4 * hi;
        if (c < dh) {
          if (a.splits > 1) {
            float *dst = a.ws + (((int64_t)sp * a.total_q + qr) * a.n_heads + head) * dh + c;
            *reinterpret_cast<float4 *>(dst) = make_float4(o[cb][4 * g], o[cb][4 * g + 1], o[cb][4 * g + 2], o[cb][4 * g + 3]);
          } else {
            T *dst = (T *)a.out + qr * a.ldo + (int64_t)head * dh + c;
            if constexpr (C::F32) {
              *reinterpret_cast<float4 *>(dst) = make_float4(o[cb][4 * g] * inv, o[cb][4 * g + 1] * inv, o[cb][4 * g + 2] * inv, o[cb][4 * g + 3] * inv);
            } else {
              bf16x4 v;
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] = (bf16_t)(o[cb][4 * g + e] * inv);
              *reinterpret_cast<bf16x4 *>(dst) = v;
            }
          }
        }
      }
  }
  if (row_ok && hi == 0) {
    const int64_t at = (int64_t)(q0 + tok) * a.n_heads + head;
    if (a.splits > 1) {
      float *dst = a.ws + (int64_t)a.splits * a.total_q * a.n_heads * dh + ((int64_t)sp * a.total_q * a.n_heads + at) * 2;
      *reinterpret_cast<float2 *>(dst) = make_float2(l_tot > 0.f ? m_run * p.sl2 : -INFINITY, l_tot);
    } else if (a.lse) {
      a.lse[at] = l_tot > 0.f ? m_run * p.sl2 * kLn2 + logf(l_tot) : -INFINITY;
    }
  }
}

// Joins the chunks of a row: out = sum 2^(m_c - m) O_c / sum 2^(m_c - m) l_c, one wave per (token, head).  Chunks behind the row's last
// key left l = 0 and no O.
template <typename T>
__global__ __launch_bounds__(256) void attn_rows_join_kernel(RowsAttn a) {
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t all = (int64_t)a.total_q * a.n_heads;
  if (id >= all) return;
  const int row = (int)(id / a.n_heads), head = (int)(id - (int64_t)row * a.n_heads), dh = a.head_dim;
  if (row < a.cu_q[0] || row >= a.cu_q[a.n_seqs]) return;
  const float2 *ml = reinterpret_cast<const float2 *>(a.ws + (int64_t)a.splits * all * dh) + id;
  float m = -INFINITY;
  for (int c = lane; c < a.splits; c += 64) m = fmaxf(m, ml[c * all].x);
  m = wave_max(m);
  const int ch = lane * 2;
  float l = 0.f, o0 = 0.f, o1 = 0.f;
  if (m > -INFINITY) {
    for (int c0 = 0; c0 < a.splits; c0 += 64) {
      float w = 0.f, lc = 0.f;
      if (c0 + lane < a.splits) {
        const float2 v = ml[(c0 + lane) * all];
        w = __builtin_amdgcn_exp2f(v.x - m);
        lc = v.y;
      }
      unsigned long long live = __builtin_amdgcn_ballot_w64(lc > 0.f);
      while (live) {
        const int i = __builtin_ctzll(live);
        live &= live - 1;
        const float wi = __shfl(w, i, kWave);
        l = fmaf(wi, __shfl(lc, i, kWave), l);
        if (ch < dh) {
          const float2 x = *reinterpret_cast<const float2 *>(a.ws + ((int64_t)(c0 + i) * all + id) * dh + ch);
          o0 = fmaf(wi, x.x, o0);
          o1 = fmaf(wi, x.y, o1);
        }
      }
    }
  }
  const float inv = l > 0.f ? 1.f / l : 0.f;
  if (ch < dh) {
    T *dst = (T *)a.out + (int64_t)row * a.ldo + (int64_t)head * dh + ch;
    dst[0] = from_f32<T>(o0 * inv);
    dst[1] = from_f32<T>(o1 * inv);
  }
  if (a.lse && lane == 0) a.lse[id] = l > 0.f ? m * kLn2 + logf(l) : -INFINITY;
}

template <typename T, int DHP, bool PAGED, int NW, int KW>
hipError_t launch_shape(const RowsAttn &a, hipStream_t s) {
  using C = Tile<T, DHP, NW, KW>;
  if (hipError_t e = allow_dynamic_lds<&attn_rows_kernel<T, DHP, PAGED, NW, KW>, C::SMEM>(); e != hipSuccess) return e;
  RowsKernelArgs p{a, a.n_heads / a.kv_heads, 0, a.scale * kLog2e};
  p.slots = (int)((int64_t)a.total_q * p.group / C::ROWS) + a.n_seqs;
  const int64_t grid = (int64_t)p.slots * a.splits * a.kv_heads;
  attn_rows_kernel<T, DHP, PAGED, NW, KW><<<dim3((unsigned)grid), 64 * C::WAVES, C::SMEM, s>>>(p);
  if (hipError_t e = hipGetLastError(); e != hipSuccess || a.splits == 1) return e;
  attn_rows_join_kernel<T><<<dim3((unsigned)(((int64_t)a.total_q * a.n_heads + 3) / 4)), 256, 0, s>>>(a);
  return hipGetLastError();
}

// Few rows per sequence on average: the key kernel.
bool few_rows(int total_q, int n_seqs, int group) { return (int64_t)total_q * group <= (int64_t)n_seqs * 32; }

template <typename T, int DHP, bool PAGED>
hipError_t launch_rows_of(const RowsAttn &a, hipStream_t s) {
  return few_rows(a.total_q, a.n_seqs, a.n_heads / a.kv_heads) ? launch_shape<T, DHP, PAGED, 1, 4>(a, s) : launch_shape<T, DHP, PAGED, 4, 1>(a, s);
}
template <typename T, bool PAGED>
hipError_t launch_dim(const RowsAttn &a, hipStream_t s) {
  if (a.head_dim <= 64) return launch_rows_of<T, 64, PAGED>(a, s);
  if (a.head_dim <= 96) return launch_rows_of<T, 96, PAGED>(a, s);
  return launch_rows_of<T, 128, PAGED>(a, s);
}

}  // namespace

RowsPlan rows_attention_plan(int dt, int total_q, int n_seqs, int n_heads, int kv_heads, int head_dim, int64_t max_kv) {
  const int group = n_heads / kv_heads;
  const bool few = few_rows(total_q, n_seqs, group);
  const int rows = few ? 32 : 128;
  // workgroups without chunks; chunks fill the chip a few times over, none shorter than four tiles' worth of keys
  const int64_t wgs = ((int64_t)total_q * group / rows + n_seqs) * kv_heads;
  const int64_t want = 1024;
  int64_t splits = (want + wgs - 1) / wgs;
  const int64_t cap = max_kv / 512 > 1 ? max_kv / 512 : 1;
  if (splits > cap) splits = cap;
  if (splits > 256) splits = 256;
  RowsPlan p{rows, (int)splits, 0};
  if (splits > 1) p.ws_bytes = (size_t)splits * total_q * n_heads * (head_dim + 2) * sizeof(float);
  return p;
}

hipError_t launch_rows_attention(const RowsAttn &a, hipStream_t s) {
  const bool paged = a.pages.table != nullptr;
  if (a.dt == DT_BF16) return paged ? launch_dim<bf16_t, true>(a, s) : launch_dim<bf16_t, false>(a, s);
  return paged ? launch_dim<float, true>(a, s) : launch_dim<float, false>(a, s);
}

}  // namespace pf
