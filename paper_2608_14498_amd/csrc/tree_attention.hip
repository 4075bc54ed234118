// Attention of drafted tokens over a cache in pages.
//
// Row i of sequence b attends to the len[b] cached tokens and to the drafted tokens that its mask
// names; softmax statistics and sums in fp32.  A row that sees nothing is 0.
//
// Per sequence and kv head the rows are (drafted token, q head of the group) pairs: N * G query rows
// read one stream of keys and values, len tokens from pages and then the drafted ones.  The work of a
// launch is the key tiles of all sequences in a row; the lengths are on the device, so each
// workgroup sums the tiles itself and takes its equal, contiguous share of them: no host value bounds
// the split, and mixed lengths load the workgroups evenly.  A share may end inside a sequence: such
// pieces leave (max, sum, unnormalised o) records, which k_tree_merge joins.
//
// Keys and values are copied straight into LDS through buffer resources whose extent is the rows that
// exist in the page (or among the drafted tokens): the rest of a tile reads as zeros.
#include "attn_common.h"
#include "device_common.h"
#include "rp_internal.h"

#include <type_traits>

namespace rp {

namespace {

constexpr float kLowest = -3.4028235e38f;

__device__ __forceinline__ int tree_len(const TreeArgs& a, int b) { return min(max(a.len[b], 0), a.table_ld << a.lg); }
__device__ __forceinline__ int tree_nodes(const TreeArgs& a, int b) {
  return a.n_nodes ? min(max(a.n_nodes[b], 0), a.N) : a.N;
}
// Drafted tokens 32 w .. 32 w + 31 that row i sees, of n.
__device__ __forceinline__ uint32_t tree_word(const TreeArgs& a, int b, int i, int w, int n) {
  const int below = i - 32 * w;  // without a mask: tokens 0 .. i
  uint32_t m = a.mask ? a.mask[((int64_t)b * a.N + i) * a.W + w] : below < 0 ? 0u : below >= 31 ? ~0u : (2u << below) - 1;
  const int there = n - 32 * w;
  return there >= 32 ? m : there <= 0 ? 0u : m & ((1u << there) - 1);
}
__device__ __forceinline__ int tree_page(const TreeArgs& a, int b, int token) {
  return min(max(a.table[(int64_t)b * a.table_ld + (token >> a.lg)], 0), a.n_pages - 1);
}

// Key tiles of KT tokens of sequence b: those of its pages, then those of its drafted tokens.
template <int KT>
__device__ __forceinline__ int tree_tiles(const TreeArgs& a, int b) {
  const int nn = tree_nodes(a, b);
  return nn == 0 ? 0 : (tree_len(a, b) + KT - 1) / KT + (nn + KT - 1) / KT;
}

// Inclusive sum over the workgroup's threads; red holds NT / 64 values.
template <int NT>
__device__ __forceinline__ int64_t tree_scan(int64_t v, int64_t* red, int64_t* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t u = __shfl_up((long long)v, o, 64);
    if (lane >= o) v += u;
  }
  __syncthreads();
  if (lane == 63) red[w] = v;
  __syncthreads();
  int64_t sum = 0, before = 0;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) {
    before += i < w ? red[i] : 0;
    sum += red[i];
  }
  *total = sum;
  return v + before;
}

// The launch's work as one row of tiles, shared out to at most `most` shares of at least `least` tiles.
// chunk > 0: each sequence is cut into shares of its own, of `chunk` tiles (the last of it may be
// smaller); else the row is cut evenly and a share may end one sequence and begin the next.
struct TreeShares {
  int64_t tiles;
  int shares, chunk;
  __device__ int64_t begin(int w) const { return tiles * w / shares; }
  __device__ int owner(int64_t u) const { return (int)(((u + 1) * shares - 1) / tiles); }
};
struct TreePiece {  // where a share begins and how many tiles it has (none: left = 0)
  int b, t;
  int64_t left;
};

// The shares that hold sequence b, for the merge, written by the one that begins it; `first`: its first tile
// in the row.
__device__ __forceinline__ void tree_note(const TreeArgs& a, const TreeShares& sh, int b, int w, int64_t first, int nt) {
  if (threadIdx.x == 0) a.held[b] = make_int2(w, sh.chunk ? w + (nt + sh.chunk - 1) / sh.chunk - 1 : sh.owner(first + nt - 1));
}

// Share w.  All threads of the workgroup call it.  Up to 64 sequences are cut into chunks of their own
// where that makes a share at most `slack` tiles longer than an even cut: a second piece costs a
// share its queries, page ids and first tiles all over again, one after the other.  4 kv heads of 128, evenly
// cut and in chunks: 8 sequences of 300 to 1000 keys 17.1 and 11.5 us, 32 of 100 to 2000 keys 25.5 and
// 22.0; 6 trees of 7 tokens over 300 keys in fp32 16.4 and 13.4.  As many shares as there are and 64 for one
// sequence (kernel + merge, one kv head): 8800 keys of 64 in fp32 16.6 + 16.2 and 13.4 + 4.8, 60000 of
// 128 in bf16 14.6 + 16.2 and 17.0 + 5.9, 8000 of them 9.8 + 7.5 and 10.4 + 5.6.
template <int NT, int KT>
__device__ __forceinline__ TreeShares tree_find(const TreeArgs& a, int most, int least, int slack, int w, TreePiece* p) {
  __shared__ int64_t red[NT / 64];
  __shared__ int at[2];
  p->b = p->t = 0;
  p->left = 0;
  auto even = [&](int64_t tiles) {
    const int64_t fit = tiles / least;
    return TreeShares{tiles, fit < 1 ? 1 : fit < most ? (int)fit : most, 0};
  };
  if (a.few) {  // every wave by itself, a sequence a lane
    const int lane = threadIdx.x & 63;
    const int mine = lane < a.B ? tree_tiles<KT>(a, lane) : 0;
    const int incl = wave_scan(mine), total = __builtin_amdgcn_readlane(incl, 63);
    TreeShares sh = even(total);
    // no more than 64 shares a sequence on the average, which a wave of the merge takes at once
    const int per = min(most, 64 * a.B), ideal = max(least, (total + per - 1) / per);
    for (int c = ideal; c <= ideal + slack && total > 0; c += 1 + c / 16) {
      const int cuts = (mine + c - 1) / c, ci = wave_scan(cuts), n = __builtin_amdgcn_readlane(ci, 63);
      if (n > most) continue;
      sh.shares = n;
      sh.chunk = c;
      const uint64_t past = __ballot(ci > w);
      if (past) {
        p->b = __builtin_ctzll(past);
        p->t = (w - __builtin_amdgcn_readlane(ci - cuts, p->b)) * c;
        p->left = min(c, __builtin_amdgcn_readlane(mine, p->b) - p->t);
      }
      return sh;
    }
    if (total == 0 || w >= sh.shares) return sh;
    const int u = (int)sh.begin(w);
    p->b = __builtin_ctzll(__ballot(incl > u));
    p->t = u - __builtin_amdgcn_readlane(incl - mine, p->b);
    p->left = sh.begin(w + 1) - u;
    return sh;
  }
  const int tid = threadIdx.x;
  int64_t sum = 0, part, incl = 0;
  int mine = 0;
  for (int base = 0; base < a.B; base += NT) {
    mine = base + tid < a.B ? tree_tiles<KT>(a, base + tid) : 0;
    tree_scan<NT>(mine, red, &part);
    sum += part;
  }
  const TreeShares sh = even(sum);
  if (sum == 0 || w >= sh.shares) return sh;
  const int64_t u = sh.begin(w);
  sum = 0;
  for (int base = 0; base < a.B && sum <= u; base += NT) {
    mine = base + tid < a.B ? tree_tiles<KT>(a, base + tid) : 0;
    incl = sum + tree_scan<NT>(mine, red, &part);
    if (incl > u && incl - mine <= u) {
      at[0] = base + tid;
      at[1] = (int)(u - (incl - mine));
    }
    sum += part;
  }
  __syncthreads();
  p->b = __builtin_amdgcn_readfirstlane(at[0]);
  p->t = __builtin_amdgcn_readfirstlane(at[1]);
  p->left = sh.begin(w + 1) - u;
  return sh;
}

// Records: share w leaves at most two, of the piece that continues a sequence (slot 0) and of the one
// that begins one it does not end (slot 1).  A record is o [rows][D], then (max in log2 units, sum)
// pairs of the block's BQ rows.
__host__ __device__ constexpr int tree_record(int BQ, int D) { return BQ * (D + 2); }
__device__ __forceinline__ int64_t tree_record_at(const TreeArgs& a, int w, int slot, int g, int rb, int RB, int BQ) {
  return ((((int64_t)w * 2 + slot) * a.Hkv + g) * RB + rb) * tree_record(BQ, a.D);
}

template <typename T16>
__device__ __forceinline__ bool not_finite(uint32_t w) {  // either half of w
  constexpr uint32_t e = std::is_same<T16, f16_t>::value ? 0x7c00u : 0x7f80u;
  return (w & e) == e || (w >> 16 & e) == e;
}
template <typename T16>
__device__ __forceinline__ uint4 flip_sign(uint4 v, uint32_t flip) {
  return make_uint4(v.x ^ flip, v.y ^ flip, v.z ^ flip, v.w ^ flip);
}

// Drafted values that are not numbers: a weight of 0 would not keep them from rows that do not see
// their token.  Rows that do see it take them here, as they are (their weight is positive);
// the tile is then cleaned of them (tree_clean) and multiplied as any other.
// vis: the tile's tokens that this lane's row sees; V rows of 8-element chunks swizzled by vswz.
template <typename T16, int D>
__device__ __forceinline__ void tree_odd_values(const T16* v, uint32_t vis, int fk, f32x16_t (&o)[D / 32]) {
  typedef Half16<T16> H;
  auto odd = [](float x, bool seen) { return seen && !(fabsf(x) <= 3.4028235e38f) ? x : 0.f; };
#pragma unroll 1
  for (int key = 0; key < 32; ++key) {
    const bool seen = vis >> key & 1;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint2 x = *reinterpret_cast<const uint2*>(v + key * D + ((db * 4 + c) ^ vswz<D>(key)) * 8 + 4 * fk);
        o[db][4 * c] += odd(H::lo_f(x.x), seen);
        o[db][4 * c + 1] += odd(H::hi_f(x.x), seen);
        o[db][4 * c + 2] += odd(H::lo_f(x.y), seen);
        o[db][4 * c + 3] += odd(H::hi_f(x.y), seen);
      }
  }
}
template <typename T16>
__device__ __forceinline__ u32x4_t tree_clean(u32x4_t x) {
  constexpr uint32_t e = std::is_same<T16, f16_t>::value ? 0x7c00u : 0x7f80u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((x[i] & e) == e) x[i] &= 0xffff0000u;
    if ((x[i] >> 16 & e) == e) x[i] &= 0xffffu;
  }
  return x;
}

// A score, or -inf where it is not seen: its weight is 0 by itself, as maxima are kLowest at least.  The
// empty asm keeps a branch around it a branch: the compiler would mask all scores of all tiles
// instead, most of which are whole.
__device__ __forceinline__ float tree_masked(float s, bool seen) {
  s = seen ? s : -__builtin_inff();
  asm volatile("" : "+v"(s));
  return s;
}

// Weights are 2^(score - m), rounded to the 16-bit type for the value product (the sum takes them unrounded): an error of
// half a step of a weight, as the output's own rounding is of the output.  fp16 has no such half steps below 2^-14 and
// nothing below 2^-25, so m is kept kLift under the row's maximum there: weights down to 2^-20 of the largest are rounded by
// half a step and smaller ones by at most 2^-31 of it, 2^-12 of the row over 2^19 keys; and with up to 2^kSlack more before
// m is raised the largest is 2^12.  (With m at the maximum 2^18 keys whose weights are 2^-25.2 of one of them lost
// their 0.6% of the row.  A slack of 4 beside a lift of 7: 320 rows over 8 x 16384 keys 1% slower; 6 and 6: no slower.)
template <typename T16>
struct TreeRange {
  static constexpr bool half = std::is_same<T16, f16_t>::value;
  static constexpr float kLift = half ? 6.f : 0.f, kSlack = half ? 6.f : kLazy;
};

// The softmax step of 32 keys for the row of this lane: s raw scores in, weights out.
// vis: the keys it sees (bit = key), where `some` (uniform) says that it may not see all.
template <typename T16, int DB>
__device__ __forceinline__ void tree_softmax(f32x16_t& s, bool some, uint32_t vis, int fk, float c2, float& m, float& l,
                                             f32x16_t (&o)[DB]) {
  if (some) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = tree_masked(s[e], vis >> (4 * fk) >> (8 * (e >> 2) + (e & 3)) & 1);
  }
  float mx = kLowest;
#pragma unroll
  for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[e]);
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
  mx = fmaf(fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])), c2, -TreeRange<T16>::kLift);
  // raised only where some lane's maximum grows by more than 2^kSlack: numerator and sum share it
  if (__any(mx > m + TreeRange<T16>::kSlack)) {
    const float mn = fmaxf(m, mx);
    const float alpha = __builtin_amdgcn_exp2f(m - mn);
    m = mn;
    l *= alpha;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[db][e] *= alpha;
  }
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    s[e] = __builtin_amdgcn_exp2f(fmaf(s[e], c2, -m));
    sum += s[e];
  }
  l += sum;
}
// Scores to log2 units.  A negative scale is a positive one on queries of the other sign; 0 is taken as a
// tiny number, as -inf times it is to stay -inf.
__device__ __forceinline__ float tree_c2(float scale) { return fmaxf(fabsf(scale) * 1.4426950408889634f, 1e-30f); }

// Four output values of a finished row.
template <typename T16>
__device__ __forceinline__ void tree_store4(T16* to, float4 v, float inv) {
  typedef Half16<T16> H;
  uint2 w;
  w.x = H::pack2(v.x * inv, v.y * inv);
  w.y = H::pack2(v.z * inv, v.w * inv);
  *reinterpret_cast<uint2*>(to) = w;
}
__device__ __forceinline__ float tree_inv(float l) { return l == 0.f ? 0.f : 1.0f / l; }

}  // namespace

// ------------------------------------------------------------------------------------
// Up to 64 rows a kv head (one token, small trees): bound by reading the cache.  A workgroup's three
// waves take the tiles of 32 keys in turn, each through an LDS ring of three stages of its own
// (two tiles of 16 KB in flight a wave; no barrier inside a piece), and join their sums in LDS at the
// piece's end.  S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_32x32x16 as in the prefix kernel:
// a lane holds one row's scores.  A wave's page ids are read 64 tiles ahead, a lane each.
// 64 x 8192 keys, 4 kv heads of 128: 193 us, 5.6 TB/s.  One tile and one sequence: 9.5 us, of which
// finding the share 3, the queries and the first tile 3, the rest mostly the fetch of code that runs
// once, as early exits show; one sequence of 4000 keys 10.7 (and 5.2 for the merge).
// ------------------------------------------------------------------------------------
constexpr int TS_WAVES = 3;
template <typename T16, int D, int QW, bool SMALL>
__device__ __forceinline__ void tree_stream(const TreeArgs& a, int shares, int least, int slack) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef Half16<T16> H;
  typedef typename H::V8 V8;
  constexpr int KT = 32, CH = D / 8, KSTEPS = D / 16, DB = D / 32, NW = TS_WAVES;
  constexpr int LOADS = KT * CH / 64;    // copies of a wave per matrix and tile
  constexpr int GL = LOADS / 4;          // of 8 keys
  constexpr int QPS = 2 * KT * CH / 64;  // 16-byte quads of a lane in one stage
  static_assert(QW * DB * 4 + 1 <= 3 * QPS, "a wave's sums fit its stages");
  __shared__ u32x4_t S0[NW][2 * KT * CH], S1[NW][2 * KT * CH], S2[NW][2 * KT * CH];  // K tile, V tile
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 31, fk = lane >> 5;
  const int g = blockIdx.x % a.Hkv, w = blockIdx.x / a.Hkv;
  const int G = a.Hq / a.Hkv;
  TreePiece pc;
  const TreeShares sh = tree_find<64 * NW, KT>(a, shares, least, slack, w, &pc);
  int b = pc.b, t0 = pc.t;
  int64_t left = pc.left;

  const uint32_t row_bytes = (uint32_t)a.Hkv * D * sizeof(T16);
  uint32_t koff[LOADS], voff[LOADS];
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    const int slot = j * 64 + lane, key = slot / CH, cp = slot % CH, from = SMALL ? key & 7 : key;
    koff[j] = (uint32_t)from * row_bytes + (uint32_t)((cp ^ kswz<D>(key)) * 16);
    voff[j] = (uint32_t)from * row_bytes + (uint32_t)((cp ^ vswz<D>(key)) * 16);
  }
  const float c2 = tree_c2(a.scale);
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
  const int tr_p = lane & 15;
  const int tr_key = fk * 4 + (tr_p >> 2);
  const int tr_col = ((lane & 16) ? 16 : 0) + 4 * (tr_p & 3);

  for (; left > 0; ++b, t0 = 0) {
    const int n0 = __builtin_amdgcn_readfirstlane(tree_len(a, b)), nn = __builtin_amdgcn_readfirstlane(tree_nodes(a, b));
    if (nn == 0) continue;
    const int P0 = (n0 + KT - 1) / KT, nt = P0 + (nn + KT - 1) / KT;
    const int t1 = __builtin_amdgcn_readfirstlane(t0 + (int)min((int64_t)(nt - t0), left)), rows = nn * G;
    if (t0 == 0 && g == 0) tree_note(a, sh, b, w, sh.chunk ? 0 : sh.begin(w + 1) - left, nt);
    left -= t1 - t0;
    // This wave's tiles are t0 + wave + NW i.  Of drafted tokens there are two tiles at most (N <= 64),
    // next to each other, so a wave has one at most: td, which it takes first, where the one copy of
    // the code for masks and odd values is.  Then its cached tiles.
    const int td = max(P0, t0) + ((wave + t0 - max(P0, t0)) % NW + NW) % NW;
    const int ahead = td < t1 ? 1 : 0;
    const int own = (min(t1, P0) - t0 - wave + NW - 1) / NW;  // cached tiles (<= 0: none)
    const int64_t row0 = (int64_t)b * a.N;
    V8 qf[QW][KSTEPS];
    uint32_t drafted[QW];
#pragma unroll
    for (int qi = 0; qi < QW; ++qi) {
      const int r = qi * 32 + fr, i = r / G;
      const bool is = r < rows;
      const T16* qp = (const T16*)a.q + (row0 + i) * a.q_ld + (g * G + r - i * G) * D + fk * 8;
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) {
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (is) v = flip_sign<T16>(*reinterpret_cast<const uint4*>(qp + ks * 16), flip);
        qf[qi][ks] = H::as_v8(v);
      }
      drafted[qi] = is && ahead ? tree_word(a, b, i, td - P0, nn) : 0u;
    }
    f32x16_t o[QW][DB];
    float m[QW], l[QW];
#pragma unroll
    for (int qi = 0; qi < QW; ++qi) {
      m[qi] = kLowest;
      l[qi] = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[qi][db][e] = 0.f;
    }

    int lead = ahead;  // the drafted tile is still to do
    for (int seg = 0; seg < own || lead; seg += 64) {
      const int n = max(0, min(64, own - seg)), ts = t0 + wave + NW * seg;  // cached tiles ts + NW i, i < n
      int pid[SMALL ? 4 : 1];
#pragma unroll
      for (int q = 0; q < (SMALL ? 4 : 1); ++q) {
        const int token = min((ts + NW * lane) * KT + 8 * q, n0 - 1);
        pid[q] = lane < n && token >= 0 ? tree_page(a, b, token) : 0;
      }
      // Copies the 32 tokens of cached tile i, or of the drafted tile (i < 0), into R; past the
      // segment's tiles nothing (out of range: nothing is fetched), so that the compiler counts the
      // copies exactly.
      auto load = [&](u32x4_t* R, int i) __attribute__((always_inline)) {
        const bool cached = i >= 0;
        const int first = cached ? (ts + NW * i) * KT : (td - P0) * KT;
        const int cnt = i < n ? min(KT, (cached ? n0 : nn) - first) : 0;
        const char* kb = (const char*)(cached ? a.k : a.kn) + (int64_t)g * D * sizeof(T16);
        const char* vb = (const char*)(cached ? a.v : a.vn) + (int64_t)g * D * sizeof(T16);
#pragma unroll
        for (int q = 0; q < (SMALL ? 4 : 1); ++q) {
          const int page = __builtin_amdgcn_readlane(pid[q], i & 63), from = first + 8 * q;
          const int64_t row = cached ? ((int64_t)page << a.lg) + (from & ((1 << a.lg) - 1)) : row0 + from;
          const int c = SMALL ? min(8, cnt - 8 * q) : cnt;
          const int ext = c > 0 ? (int)((uint32_t)(c - 1) * row_bytes + D * (uint32_t)sizeof(T16)) : 0;
          const __amdgpu_buffer_rsrc_t rk =
              __builtin_amdgcn_make_buffer_rsrc(uniform_ptr((void*)(kb + row * row_bytes)), 0, __builtin_amdgcn_readfirstlane(ext), 0x00020000);
          const __amdgpu_buffer_rsrc_t rv =
              __builtin_amdgcn_make_buffer_rsrc(uniform_ptr((void*)(vb + row * row_bytes)), 0, __builtin_amdgcn_readfirstlane(ext), 0x00020000);
#pragma unroll
          for (int j = q * GL; j < (SMALL ? (q + 1) * GL : LOADS); ++j) {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_void_t*)(R + j * 64), 16, koff[j], 0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_void_t*)(R + KT * CH + j * 64), 16, voff[j], 0, 0, 0);
          }
        }
      };
      // FIRST: the tile that may be the drafted one.
      auto tile = [&](u32x4_t* R, int i, auto first_) __attribute__((always_inline)) {
        constexpr bool FIRST = decltype(first_)::value;
        u32x4_t *Kc = R, *Vc = R + KT * CH;
        f32x16_t s[QW];
        V8 kf[KSTEPS];  // (read at once: the compiler would wait for each)
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks) kf[ks] = __builtin_bit_cast(V8, Kc[fr * CH + ((ks * 2 + fk) ^ kswz<D>(fr))]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int ks = 0; ks < KSTEPS; ++ks)
#pragma unroll
          for (int qi = 0; qi < QW; ++qi) s[qi] = H::mma(kf[ks], qf[qi][ks], ks == 0 ? f32x16_t{} : s[qi]);
        // s[qi][0][e] = score(key 8(e/4) + 4 fk + e%4, row fr)
        const bool cached = !FIRST || i >= 0;
        const int there = n0 - (ts + NW * i) * KT;
        const uint32_t tail = there >= KT ? ~0u : (1u << (there & 31)) - 1;
        const T16* vbase = reinterpret_cast<const T16*>(Vc);
#pragma unroll
        for (int qi = 0; qi < QW; ++qi)
          tree_softmax<T16, DB>(s[qi], !cached || there < KT, cached ? tail : drafted[qi], fk, c2, m[qi], l[qi], o[qi]);
        if (!cached) {
          bool odd = false;
#pragma unroll
          for (int j = 0; j < LOADS; ++j) {
            const u32x4_t x = Vc[j * 64 + lane];
            odd |= not_finite<T16>(x[0]) || not_finite<T16>(x[1]) || not_finite<T16>(x[2]) || not_finite<T16>(x[3]);
          }
          if (__any(odd)) {
#pragma unroll
            for (int qi = 0; qi < QW; ++qi) tree_odd_values<T16, D>(vbase, drafted[qi], fk, o[qi]);
#pragma unroll
            for (int j = 0; j < LOADS; ++j) Vc[j * 64 + lane] = tree_clean<T16>(Vc[j * 64 + lane]);
          }
        }
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          V8 pf[QW];
#pragma unroll
          for (int qi = 0; qi < QW; ++qi) {
            const f32x16_t& x = s[qi];
            pf[qi] = H::as_v8(make_uint4(H::pack2(x[hh * 8 + 0], x[hh * 8 + 1]), H::pack2(x[hh * 8 + 2], x[hh * 8 + 3]),
                                         H::pack2(x[hh * 8 + 4], x[hh * 8 + 5]), H::pack2(x[hh * 8 + 6], x[hh * 8 + 7])));
          }
          const int ka = hh * 16 + tr_key, kc = ka + 8;
#pragma unroll
          for (int db = 0; db < DB; ++db) {
            const int col = db * 32 + tr_col;
            const int ca = ((col >> 3) ^ vswz<D>(ka)) * 8 + (col & 7);
            const int cc = ((col >> 3) ^ vswz<D>(kc)) * 8 + (col & 7);
            const v4i16_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t*)(vbase + ka * D + ca));
            const v4i16_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t*)(vbase + kc * D + cc));
            const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
            const V8 vf = H::as_v8(make_uint4(l2.x, l2.y, h2.x, h2.y));
#pragma unroll
            for (int qi = 0; qi < QW; ++qi) o[qi][db] = H::mma(vf, pf[qi], o[qi][db]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      };
      // Tile i is in stage (i + lead) % 3, refilled once read.  The first before the loop: its wait covers
      // the register loads too (a loop entered with some pending would drain every copy).
      const std::true_type first{};
      const std::false_type later{};
      const int i0 = -lead;
      load(S0[wave], i0);
      load(S1[wave], i0 + 1);
      load(S2[wave], i0 + 2);
      tile(S0[wave], i0, first);
      load(S0[wave], i0 + 3);
      for (int i = i0 + 1; i < n; i += 3) {
        tile(S1[wave], i, later);
        load(S1[wave], i + 3);
        if (i + 1 < n) tile(S2[wave], i + 1, later);
        load(S2[wave], i + 4);
        if (i + 2 < n) tile(S0[wave], i + 2, later);
        load(S0[wave], i + 5);
      }
      __builtin_amdgcn_s_waitcnt(0);  // the stages are free
      lead = 0;
    }

    // ---- the waves' sums joined: quad k = (qi, db, c) holds dims db*32 + 8 c + 4 fk .. + 3 of row qi*32 + fr ----
    auto quad = [&](int wv, int k) -> u32x4_t* {
      u32x4_t* st = k < QPS ? S0[wv] : k < 2 * QPS ? S1[wv] : S2[wv];
      return st + (k % QPS) * 64 + lane;
    };
#pragma unroll
    for (int qi = 0; qi < QW; ++qi)
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float4 v = make_float4(o[qi][db][4 * c], o[qi][db][4 * c + 1], o[qi][db][4 * c + 2], o[qi][db][4 * c + 3]);
          *quad(wave, (qi * DB + db) * 4 + c) = __builtin_bit_cast(u32x4_t, v);
        }
    {
      float4 v = make_float4(m[0], l[0], 0.f, 0.f);
      if constexpr (QW == 2) {
        v.z = m[1];
        v.w = l[1];
      }
      *quad(wave, QW * DB * 4) = __builtin_bit_cast(u32x4_t, v);
    }
    __syncthreads();
    float f[QW][NW], M[QW], L[QW];
#pragma unroll
    for (int qi = 0; qi < QW; ++qi) {
      float mw[NW], lw[NW];
      M[qi] = kLowest;
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        const float4 x = __builtin_bit_cast(float4, *quad(v, QW * DB * 4));
        mw[v] = qi ? x.z : x.x;
        lw[v] = qi ? x.w : x.y;
        M[qi] = fmaxf(M[qi], mw[v]);
      }
      L[qi] = 0.f;
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        f[qi][v] = __builtin_amdgcn_exp2f(mw[v] - M[qi]);
        L[qi] = fmaf(lw[v], f[qi][v], L[qi]);
      }
      L[qi] += __shfl_xor(L[qi], 32, kWave);
    }
    const bool whole = t0 == 0 && t1 == nt;
    float* rec = a.part + tree_record_at(a, w, t0 == 0, g, 0, 1, 32 * QW);
    for (int k = wave; k < QW * DB * 4; k += NW) {
      const int qi = k / (DB * 4), dim = (k % (DB * 4)) / 4 * 32 + 8 * (k & 3) + 4 * fk, r = qi * 32 + fr;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        const float4 y = __builtin_bit_cast(float4, *quad(v, k));
        const float z = QW == 2 && qi ? f[QW - 1][v] : f[0][v];
        x.x = fmaf(y.x, z, x.x);
        x.y = fmaf(y.y, z, x.y);
        x.z = fmaf(y.z, z, x.z);
        x.w = fmaf(y.w, z, x.w);
      }
      if (r >= rows) continue;
      if (whole) {
        const int i = r / G;
        tree_store4<T16>((T16*)a.out + ((row0 + i) * a.Hq + g * G + r - i * G) * D + dim, x, tree_inv(QW == 2 && qi ? L[QW - 1] : L[0]));
      } else {
        *reinterpret_cast<float4*>(rec + r * D + dim) = x;
      }
    }
    if (!whole && wave == 0 && fk == 0) {
#pragma unroll
      for (int qi = 0; qi < QW; ++qi)
        if (qi * 32 + fr < rows) *reinterpret_cast<float2*>(rec + 32 * QW * D + 2 * (qi * 32 + fr)) = make_float2(M[qi], L[qi]);
    }
    __syncthreads();  // the stages are free again
  }
#endif
}

// (One wave a SIMD could have 512 registers, but half of them only by way of moves: 32 rows stay in 256.)
template <typename T16, int D, bool SMALL>
__global__ __launch_bounds__(64 * TS_WAVES) __attribute__((amdgpu_num_vgpr(256))) void k_tree_stream32(TreeArgs a, int shares, int least, int slack) {
  tree_stream<T16, D, 1, SMALL>(a, shares, least, slack);
}
template <typename T16, int D, bool SMALL>
__global__ __launch_bounds__(64 * TS_WAVES) void k_tree_stream64(TreeArgs a, int shares, int least, int slack) {
  tree_stream<T16, D, 2, SMALL>(a, shares, least, slack);
}

// ------------------------------------------------------------------------------------
// More rows (large trees).  A workgroup's four waves hold 32 rows each and share tiles of 32 keys in a ring
// of four stages; two workgroups share a CU.  One barrier a tile: behind it the tile has landed for every
// wave and the one before has been read by all, so its stage takes the copies of the tile three further
// on.  The K fragments are read all at once (the compiler would wait for each), V's during the softmax.
//
// 112 rows over 32 x 8192 keys: 129 us, 4.2 TB/s, near what the copies alone take.  448 rows over 8 x
// 16384: 168 us, 0.72 PFLOP/s, where a SIMD's two waves spend 45% of the time on products and 41% on
// the softmax, hardly at once.  Tried and left: 64 rows a wave (the sums spill); eight waves a barrier (all
// wait for the slowest: 10% slower); tiles of 64 keys (two stages fit two workgroups: the copies come
// too late); scores a tile ahead (no gain); eight waves of 32 rows in two groups half a tile apart,
// one at the products while the other is at the softmax (448 rows 161 us, but 320 rows 300 instead of 262: the
// second block of 256 is filled to a quarter).
// ------------------------------------------------------------------------------------
template <int N>
__device__ __forceinline__ void tree_ring_step() {  // this wave's copies but the last N have landed; all waves are here
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

template <typename T16, int D>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
void k_tree_block(TreeArgs a, int shares, int least, int slack, int RB) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef Half16<T16> H;
  typedef typename H::V8 V8;
  constexpr int NW = 4, BQ = NW * 32, KT = 32, NS = 4, CH = D / 8, KSTEPS = D / 16, DB = D / 32;
  constexpr int LOADS = KT * CH / (NW * 64), KW = KT / NW;  // a wave copies KW keys of a tile
  static_assert(KW <= 8 && LOADS * 64 == KW * CH, "a wave's keys lie in one page");
  __shared__ u32x4_t S0[2 * KT * CH], S1[2 * KT * CH], S2[2 * KT * CH], S3[2 * KT * CH];  // K tile, V tile
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 31, fk = lane >> 5;
  const int G = a.Hq / a.Hkv;
  // the row blocks of one share next to each other on one XCD: its L2 serves all but the first
  const int local = blockIdx.x >> 3, pair = local / RB * 8 + (blockIdx.x & 7), rb = local % RB;
  const int g = pair % a.Hkv, w = pair / a.Hkv;
  if (w >= shares) return;
  TreePiece pc;
  const TreeShares sh = tree_find<64 * NW, KT>(a, shares, least, slack, w, &pc);
  int b = pc.b, t0 = pc.t;
  int64_t left = pc.left;

  const uint32_t row_bytes = (uint32_t)a.Hkv * D * sizeof(T16);
  uint32_t koff[LOADS], voff[LOADS];
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    const int slot = (wave * LOADS + j) * 64 + lane, key = slot / CH, cp = slot % CH, from = key - wave * KW;
    koff[j] = (uint32_t)from * row_bytes + (uint32_t)((cp ^ kswz<D>(key)) * 16);
    voff[j] = (uint32_t)from * row_bytes + (uint32_t)((cp ^ vswz<D>(key)) * 16);
  }
  const float c2 = tree_c2(a.scale);
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
  const int tr_p = lane & 15;
  const int tr_key = fk * 4 + (tr_p >> 2);
  const int tr_col = ((lane & 16) ? 16 : 0) + 4 * (tr_p & 3);

  for (; left > 0; ++b, t0 = 0) {
    const int n0 = __builtin_amdgcn_readfirstlane(tree_len(a, b)), nn = __builtin_amdgcn_readfirstlane(tree_nodes(a, b));
    if (nn == 0) continue;
    const int P0 = (n0 + KT - 1) / KT, nt = P0 + (nn + KT - 1) / KT;
    const int t1 = __builtin_amdgcn_readfirstlane(t0 + (int)min((int64_t)(nt - t0), left)), rows = nn * G;
    if (t0 == 0 && g == 0 && rb == 0) tree_note(a, sh, b, w, sh.chunk ? 0 : sh.begin(w + 1) - left, nt);
    left -= t1 - t0;
    if (rb * BQ >= rows) continue;
    const int64_t row0 = (int64_t)b * a.N;
    const int r = rb * BQ + wave * 32 + fr, ri = min(r, rows - 1) / G;  // (rows past the last repeat it)
    V8 qf[KSTEPS];
    {
      const T16* qp = (const T16*)a.q + (row0 + ri) * a.q_ld + (g * G + min(r, rows - 1) - ri * G) * D + fk * 8;
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) qf[ks] = H::as_v8(flip_sign<T16>(*reinterpret_cast<const uint4*>(qp + ks * 16), flip));
    }
    f32x16_t o[DB];
    float m = kLowest, l = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[db][e] = 0.f;

    // s[e] = score(key 8(e/4) + 4 fk + e%4 of the tile in R, row fr)
    auto read_k = [&](const u32x4_t* R, V8 (&kf)[KSTEPS]) __attribute__((always_inline)) {
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) kf[ks] = __builtin_bit_cast(V8, R[fr * CH + ((ks * 2 + fk) ^ kswz<D>(fr))]);
    };
    auto scores = [&](const V8 (&kf)[KSTEPS], f32x16_t& s) __attribute__((always_inline)) {
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) s = H::mma(kf[ks], qf[ks], ks == 0 ? f32x16_t{} : s);
    };
    // o += V^T P^T
    auto read_v = [&](const u32x4_t* R, V8 (&vf)[2 * DB]) __attribute__((always_inline)) {
      const T16* vbase = reinterpret_cast<const T16*>(R + KT * CH);
#pragma unroll
      for (int i = 0; i < 2 * DB; ++i) {
        const int ka = i / DB * 16 + tr_key, kc = ka + 8, col = i % DB * 32 + tr_col;
        const int ca = ((col >> 3) ^ vswz<D>(ka)) * 8 + (col & 7);
        const int cc = ((col >> 3) ^ vswz<D>(kc)) * 8 + (col & 7);
        const v4i16_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t*)(vbase + ka * D + ca));
        const v4i16_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_t*)(vbase + kc * D + cc));
        const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
        vf[i] = H::as_v8(make_uint4(l2.x, l2.y, h2.x, h2.y));
      }
    };
    auto values = [&](const V8 (&vf)[2 * DB], const f32x16_t& x) __attribute__((always_inline)) {
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const V8 pf = H::as_v8(make_uint4(H::pack2(x[hh * 8 + 0], x[hh * 8 + 1]), H::pack2(x[hh * 8 + 2], x[hh * 8 + 3]),
                                          H::pack2(x[hh * 8 + 4], x[hh * 8 + 5]), H::pack2(x[hh * 8 + 6], x[hh * 8 + 7])));
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] = H::mma(vf[hh * DB + db], pf, o[db]);
      }
    };
    // Drafted tile d from R, whole.
    auto draft = [&](u32x4_t* R, int d) __attribute__((always_inline)) {
      f32x16_t s;
      V8 kf[KSTEPS], vf[2 * DB];
      read_k(R, kf);
      scores(kf, s);
      const uint32_t vis = tree_word(a, b, ri, d, nn);
      tree_softmax<T16, DB>(s, true, vis, fk, c2, m, l, o);
      u32x4_t* Vc = R + KT * CH;
      bool odd = false;  // (every wave looks at the whole tile, so that all of them agree)
#pragma unroll 2
      for (int j = 0; j < KT * CH / 64; ++j) {
        const u32x4_t x = Vc[j * 64 + lane];
        odd |= not_finite<T16>(x[0]) || not_finite<T16>(x[1]) || not_finite<T16>(x[2]) || not_finite<T16>(x[3]);
      }
      if (__any(odd)) {
        tree_odd_values<T16, D>(reinterpret_cast<const T16*>(Vc), vis, fk, o);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < LOADS; ++j) Vc[(wave * LOADS + j) * 64 + lane] = tree_clean<T16>(Vc[(wave * LOADS + j) * 64 + lane]);
        __syncthreads();
      }
      read_v(R, vf);
      values(vf, s);
    };
    // Copies this wave's KW of the tokens from `first` on, of n (cached: in page `page`).
    auto copy = [&](u32x4_t* R, bool cached, int first, int n, int page) __attribute__((always_inline)) {
      const int from = first + wave * KW, c = min(KW, n - from);
      const int64_t row = cached ? ((int64_t)page << a.lg) + (from & ((1 << a.lg) - 1)) : row0 + from;
      const int64_t at = row * row_bytes + (int64_t)g * D * sizeof(T16);
      const int ext = c > 0 ? (int)((uint32_t)(c - 1) * row_bytes + D * (uint32_t)sizeof(T16)) : 0;
      const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(
          uniform_ptr((void*)((const char*)(cached ? a.k : a.kn) + at)), 0, __builtin_amdgcn_readfirstlane(ext), 0x00020000);
      const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(
          uniform_ptr((void*)((const char*)(cached ? a.v : a.vn) + at)), 0, __builtin_amdgcn_readfirstlane(ext), 0x00020000);
#pragma unroll
      for (int j = 0; j < LOADS; ++j) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lds_void_t*)(R + (wave * LOADS + j) * 64), 16, koff[j], 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lds_void_t*)(R + KT * CH + (wave * LOADS + j) * 64), 16, voff[j], 0, 0, 0);
      }
    };
    // Cached tiles in segments of 128, whose page ids a wave holds two a lane.  Tile k of a segment is in
    // stage (k + 1) % NS.  Drafted tiles come first, in stage 0, with the first cached ones on their way.
    const int te = min(t1, P0);
    int drafts = t1 - max(t0, P0);
    for (int from = t0; from < te || drafts > 0; from += 128) {
      const int n = min(te - from, 128);
      const int work = rb * BQ + wave * 32 < rows ? n : 0;  // a wave past the last row only copies
      int pid[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int token = min((from + 64 * h + lane) * KT + wave * KW, n0 - 1);
        pid[h] = 64 * h + lane < n && token >= 0 ? tree_page(a, b, token) : 0;
      }
      auto load = [&](u32x4_t* R, int k) __attribute__((always_inline)) {  // (past the segment: nothing is fetched)
        const int p0 = __builtin_amdgcn_readlane(pid[0], k & 63), p1 = __builtin_amdgcn_readlane(pid[1], k & 63);
        copy(R, true, (from + k) * KT, k < n ? n0 : 0, k < 64 ? p0 : p1);
      };
      __syncthreads();  // the stages are free
      if (drafts > 0) copy(S0, false, (max(t0, P0) - P0) * KT, nn, 0);
      load(S1, 0);
      load(S2, 1);
      load(S3, 2);
      if (drafts > 0) {
        tree_ring_step<(NS - 1) * 2 * LOADS>();
        int d = max(t0, P0) - P0;
        for (;;) {
          draft(S0, d);
          if (--drafts <= 0) break;
          ++d;
          __syncthreads();
          copy(S0, false, d * KT, nn, 0);
          tree_ring_step<0>();
        }
      }
      // Tile k; false behind the last.  (No branch around the copies, whose issue goes between the products; the
      // compiler counts them exactly.)
      auto step = [&](u32x4_t* next, const u32x4_t* now, int k) __attribute__((always_inline)) {
        tree_ring_step<(NS - 2) * 2 * LOADS>();
        V8 kf[KSTEPS], vf[2 * DB];
        read_k(now, kf);
        __builtin_amdgcn_sched_barrier(0);
        load(next, k + NS - 1);
        if (k < work) {
          f32x16_t s;
          scores(kf, s);
          read_v(now, vf);
          const int there = n0 - (from + k) * KT;
          tree_softmax<T16, DB>(s, there < KT, (1u << (there & 31)) - 1, fk, c2, m, l, o);
          values(vf, s);
        }
      };
      for (int k = 0; k < n; k += NS) {
        step(S0, S1, k);
        step(S1, S2, k + 1);
        step(S2, S3, k + 2);
        step(S3, S0, k + 3);
      }
      __builtin_amdgcn_s_waitcnt(0);
    }

    // o[db][e] = O^T(dim db*32 + 8(e/4) + 4 fk + e%4, row r)
    const float L = l + __shfl_xor(l, 32, kWave);
    if (r < rows) {
      const bool whole = t0 == 0 && t1 == nt;
      float* rec = a.part + tree_record_at(a, w, t0 == 0, g, rb, RB, BQ);
      T16* op = (T16*)a.out + ((row0 + ri) * a.Hq + g * G + r - ri * G) * D;
      const int in = r - rb * BQ;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float4 v = make_float4(o[db][4 * c], o[db][4 * c + 1], o[db][4 * c + 2], o[db][4 * c + 3]);
          const int dim = db * 32 + 8 * c + 4 * fk;
          if (whole)
            tree_store4<T16>(op + dim, v, tree_inv(L));
          else
            *reinterpret_cast<float4*>(rec + in * D + dim) = v;
        }
      if (!whole && fk == 0) *reinterpret_cast<float2*>(rec + BQ * D + 2 * in) = make_float2(m, L);
    }
  }
#endif
}

// ------------------------------------------------------------------------------------
// fp32 on the fp32 matrix cores (v_mfma_f32_32x32x2: exact products), blocks of 32 rows whose NW waves
// take the tiles of 32 keys in turn, fragments straight from global memory as in the prefix's fp32
// kernel, and join their sums in LDS.  6 trees of 7 tokens over up to 577 keys (64): 10.0 us, a chain of
// loads (lengths, page ids, K, V) and 64 products of 64 cycles; 16 trees of 20 tokens over 3000 to 4000 keys
// (128): 73 us, 47 TFLOP/s.
// ------------------------------------------------------------------------------------
template <int D, int NW>
__global__ __launch_bounds__(NW * 64) void k_tree_f32(TreeArgs a, int shares, int least, int slack, int RB) {
  constexpr int KT = 32, NC = D / 8, DB = D / 32;
  __shared__ float4 part[NW][DB * 4][64];
  __shared__ float2 ml[NW][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int fr = lane & 31, fk = lane >> 5;
  const int G = a.Hq / a.Hkv;
  const int rb = blockIdx.x % RB, g = blockIdx.x / RB % a.Hkv, w = blockIdx.x / RB / a.Hkv;
  TreePiece pc;
  const TreeShares sh = tree_find<64 * NW, KT>(a, shares, least, slack, w, &pc);
  int b = pc.b, t0 = pc.t;
  int64_t left = pc.left;
  const int64_t ld = (int64_t)a.Hkv * D;

  for (; left > 0; ++b, t0 = 0) {
    const int n0 = __builtin_amdgcn_readfirstlane(tree_len(a, b)), nn = __builtin_amdgcn_readfirstlane(tree_nodes(a, b));
    if (nn == 0) continue;
    const int P0 = (n0 + KT - 1) / KT, nt = P0 + (nn + KT - 1) / KT;
    const int t1 = __builtin_amdgcn_readfirstlane(t0 + (int)min((int64_t)(nt - t0), left)), rows = nn * G;
    if (t0 == 0 && g == 0 && rb == 0) tree_note(a, sh, b, w, sh.chunk ? 0 : sh.begin(w + 1) - left, nt);
    left -= t1 - t0;
    if (rb * 32 >= rows) continue;
    const int64_t row0 = (int64_t)b * a.N;
    const int r = rb * 32 + fr, rc = min(r, rows - 1), ri = rc / G;
    float4 q[NC];
    const float* qp = (const float*)a.q + (row0 + ri) * a.q_ld + (g * G + rc - ri * G) * D + 4 * fk;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      q[j] = *reinterpret_cast<const float4*>(qp + 8 * j);
      q[j] = make_float4(q[j].x * a.scale, q[j].y * a.scale, q[j].z * a.scale, q[j].w * a.scale);
    }
    // page of key fr of tile t (its last one past the end), and rows' places: lane 8 j holds the
    // page of keys 8 j .. 8 j + 7
    auto page_of = [&](int t) { return t < P0 ? tree_page(a, b, min(t * KT + fr, n0 - 1)) : 0; };
    float4 kf[NC];
    auto load_k = [&](int t, int page) {
      const bool cached = t < P0;
      const int first = cached ? t * KT : (t - P0) * KT, key = min(fr, (cached ? n0 : nn) - first - 1);
      const int64_t row = cached ? ((int64_t)page << a.lg) + ((first + key) & ((1 << a.lg) - 1)) : row0 + first + key;
      const float* kp = (const float*)(cached ? a.k : a.kn) + row * ld + g * D + 4 * fk;
#pragma unroll
      for (int j = 0; j < NC; ++j) kf[j] = *reinterpret_cast<const float4*>(kp + 8 * j);
    };
    f32x16_t o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[db][e] = 0.f;
    float m = kLowest, l = 0.f;
    int page = 0, page_next = 0;
    if (t0 + wave < t1) {
      page = page_of(t0 + wave);
      if (t0 + wave + NW < t1) page_next = page_of(t0 + wave + NW);
      load_k(t0 + wave, page);
    }
    for (int t = t0 + wave; t < t1; t += NW) {
      const bool cached = t < P0;
      const int first = cached ? t * KT : (t - P0) * KT, cnt = min(KT, (cached ? n0 : nn) - first);
      uint32_t vis = cnt >= 32 ? ~0u : (1u << cnt) - 1;
      if (!cached) vis = tree_word(a, b, ri, t - P0, nn);
      float vf[DB][16];
      const float* vb = (const float*)(cached ? a.v : a.vn) + g * D;
      // Row of key 8 j: keys 8 j .. 8 j + 7 lie in one page, lane 8 j's.  (A lane's own choice is made among rows, not
      // among lanes to ask for a page.)  Past the last key the first one is read, and not used.
      int64_t at[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        at[j] = cached ? ((int64_t)__builtin_amdgcn_readlane(page, 8 * j) << a.lg) + ((first + 8 * j) & ((1 << a.lg) - 1)) : row0 + first + 8 * j;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int in = 4 * fk + (e & 3), key = 8 * (e >> 2) + in;
        const bool is = key < cnt;
        const float* vp = vb + ((is ? at[e >> 2] : at[0]) + (is ? in : 0)) * ld + fr;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const float x = vp[db * 32];
          vf[db][e] = is ? x : 0.f;
        }
      }
      f32x16_t s;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[j].x, q[j].x, s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[j].y, q[j].y, s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[j].z, q[j].z, s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(kf[j].w, q[j].w, s, 0, 0, 0);
      }
      if (t + NW < t1) load_k(t + NW, page_next);
      const uint32_t mine = vis >> (4 * fk);  // s[e]: key 8(e/4) + 4 fk + e%4
      float mx = kLowest;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[e] = mine >> (8 * (e >> 2) + (e & 3)) & 1 ? s[e] : kLowest;
        mx = fmaxf(mx, s[e]);
      }
      mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
      const float mn = fmaxf(m, mx), alpha = expf(m - mn);
      m = mn;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[db][e] *= alpha;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[e] = mine >> (8 * (e >> 2) + (e & 3)) & 1 ? expf(s[e] - mn) : 0.f;
        l += s[e];
      }
      bool odd = false;  // values that a weight of 0 would not keep away
      if (!cached) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
          for (int db = 0; db < DB; ++db) odd |= !(fabsf(vf[db][e]) <= 3.4028235e38f);
      }
      if (__any(odd)) {  // (as in tree_odd_values)
#pragma unroll 1
        for (int key = 0; key < cnt; ++key) {
          const bool seen = vis >> key & 1;
          const float* vp = (const float*)a.vn + (row0 + first + key) * ld + g * D + 4 * fk;
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int c = 0; c < 16; ++c) {
              const float x = vp[db * 32 + 8 * (c >> 2) + (c & 3)];
              o[db][c] += seen && !(fabsf(x) <= 3.4028235e38f) ? x : 0.f;
            }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
          for (int db = 0; db < DB; ++db) vf[db][e] = fabsf(vf[db][e]) <= 3.4028235e38f ? vf[db][e] : 0.f;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e)
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf[db][e], s[e], o[db], 0, 0, 0);
      page = page_next;
      if (t + 2 * NW < t1) page_next = page_of(t + 2 * NW);
    }
    l += __shfl_xor(l, 32, kWave);
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        part[wave][db * 4 + c][lane] = make_float4(o[db][4 * c], o[db][4 * c + 1], o[db][4 * c + 2], o[db][4 * c + 3]);
    ml[wave][lane] = make_float2(m, l);
    __syncthreads();
    float M = kLowest, L = 0.f, f[NW];
#pragma unroll
    for (int v = 0; v < NW; ++v) M = fmaxf(M, ml[v][lane].x);
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      f[v] = expf(ml[v][lane].x - M);
      L = fmaf(ml[v][lane].y, f[v], L);
    }
    const bool whole = t0 == 0 && t1 == nt;
    float* rec = a.part + tree_record_at(a, w, t0 == 0, g, rb, RB, 32);
    const float inv = tree_inv(L);
    for (int k = wave; k < DB * 4; k += NW) {
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        const float4 y = part[v][k][lane];
        x.x = fmaf(y.x, f[v], x.x);
        x.y = fmaf(y.y, f[v], x.y);
        x.z = fmaf(y.z, f[v], x.z);
        x.w = fmaf(y.w, f[v], x.w);
      }
      if (r >= rows) continue;
      const int dim = (k >> 2) * 32 + 8 * (k & 3) + 4 * fk;
      if (whole)
        *reinterpret_cast<float4*>((float*)a.out + ((row0 + ri) * a.Hq + g * G + r - ri * G) * D + dim) =
            make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
      else
        *reinterpret_cast<float4*>(rec + fr * D + dim) = x;
    }
    // (the fp32 kernel's maxima are natural logarithms: to log2 units for the merge)
    if (!whole && wave == 0 && fk == 0 && r < rows)
      *reinterpret_cast<float2*>(rec + 32 * D + 2 * fr) = make_float2(fmaxf(M * 1.4426950408889634f, kLowest), L);
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------
// Joins the records of the sequences that several shares hold; zeroes the padding rows where asked.
// Bound by latency (which shares, their maxima and sums, their o: three loads in a row), so a wave has
// many of each in flight.  Few rows (one sequence in many shares): a wave a row, its halves taking
// every other record.  Many rows (few shares each): eight rows a wave, a lane for each of their
// maxima, each half taking every other row.  One and eight rows a wave: 28 rows of 42 records 5.2 and 17 us,
// 280 of 64 7.6 and 18.8, 1792 of one 5.0 and 4.8, 3584 of two to five 12.5 and 8.3, 20480 of four 21.8 and 11.2.
// ------------------------------------------------------------------------------------
constexpr int TM_WAVES = 4, TM_MANY = 8;
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(64 * TM_WAVES) void k_tree_merge(TreeArgs a, int BQ, int RB) {
  constexpr int PER = D / 32;
  typedef float vec_t __attribute__((ext_vector_type(PER)));
  const int lane = threadIdx.x & 63, half = lane >> 5, at = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int G = a.Hq / a.Hkv, groups = (a.N * G + TM_WAVES * ROWS - 1) / (TM_WAVES * ROWS);
  const int r0 = (blockIdx.x % groups * TM_WAVES + wave) * ROWS, g = blockIdx.x / groups % a.Hkv, b = blockIdx.x / groups / a.Hkv;
  const int2 held = a.held[b];  // (of a sequence without rows: whatever, and not used)
  const int rows = tree_nodes(a, b) * G;
  auto out_at = [&](int r) {
    const int i = r / G;
    return (T*)a.out + (((int64_t)b * a.N + i) * a.Hq + g * G + r - i * G) * D + at * PER;
  };
  if (a.zero_rest) {
    for (int r = max(r0, rows) + half; r < min(r0 + ROWS, a.N * G); r += 2) {
#pragma unroll
      for (int c = 0; c < PER; ++c) stf(out_at(r) + c, 0.f);
    }
  }
  if (r0 >= rows) return;
  const int wa = __builtin_amdgcn_readfirstlane(held.x), wb = __builtin_amdgcn_readfirstlane(held.y);
  if (wa == wb) return;  // one share held it all
  auto record = [&](int w, int rb) { return a.part + tree_record_at(a, w, w == wa, g, rb, RB, BQ); };
  if constexpr (ROWS == 1) {
    auto across = [&](float x, auto f) {  // f over the wave, in lane moves and four reads of lanes
      x = f(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0xB1, 0xf, 0xf, false)));   // quad_perm 1,0,3,2
      x = f(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x4E, 0xf, 0xf, false)));   // quad_perm 2,3,0,1
      x = f(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x124, 0xf, 0xf, false)));  // row_ror 4
      x = f(x, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x128, 0xf, 0xf, false)));  // row_ror 8
      auto row = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), l)); };
      return f(f(row(0), row(16)), f(row(32), row(48)));
    };
    const int rb = r0 / BQ, in = r0 - rb * BQ;
    float M = kLowest, L = 0.f;
    vec_t o = {};
    for (int base = wa; base <= wb; base += 64) {
      float2 x = make_float2(kLowest, 0.f);
      if (base + lane <= wb) x = *reinterpret_cast<const float2*>(record(base + lane, rb) + BQ * D + 2 * in);
      const float mn = fmaxf(M, across(x.x, [](float p, float q) { return fmaxf(p, q); })), old = __builtin_amdgcn_exp2f(M - mn);
      const float f = __builtin_amdgcn_exp2f(x.x - mn);
      M = mn;
      L = fmaf(x.y, f, L * old);
      o *= old;
      const int n = min(64, wb - base + 1);
      for (int k = 0; k < n; k += 16) {
        vec_t v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {  // (past the last: once more the last, with weight 0)
          const int e = min(k + 2 * j + half, n - 1);
          v[j] = *reinterpret_cast<const vec_t*>(record(base + e, rb) + in * D + at * PER);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int e = k + 2 * j + half;
          const float z = __shfl(f, min(e, 63), kWave);
          o += v[j] * (e < n ? z : 0.f);
        }
      }
    }
    const float inv = tree_inv(across(L, [](float p, float q) { return p + q; }));
#pragma unroll
    for (int c = 0; c < PER; ++c) {
      const float y = (o[c] + __shfl_xor(o[c], 32, kWave)) * inv;
      if (half == 0) stf(out_at(r0) + c, y);
    }
  } else {
    static_assert(ROWS == 8, "eight rows by eight records a lane each");
    // lane (j, e) holds the maximum and sum of row r0 + j in record e of eight
    const int j8 = lane >> 3, e8 = lane & 7;
    const int rj = min(r0 + j8, rows - 1), rbj = rj / BQ, inj = rj - rbj * BQ;
    float M = kLowest, L = 0.f;
    vec_t o[ROWS / 2] = {};
    for (int base = wa; base <= wb; base += 8) {
      float2 x = make_float2(kLowest, 0.f);
      if (base + e8 <= wb) x = *reinterpret_cast<const float2*>(record(base + e8, rbj) + BQ * D + 2 * inj);
      float mn = x.x;
#pragma unroll
      for (int s = 1; s < 8; s <<= 1) mn = fmaxf(mn, __shfl_xor(mn, s, kWave));
      mn = fmaxf(M, mn);
      const float old = __builtin_amdgcn_exp2f(M - mn), f = __builtin_amdgcn_exp2f(x.x - mn);
      M = mn;
      L = fmaf(x.y, f, L * old);
      const int n = min(8, wb - base + 1);
#pragma unroll
      for (int p = 0; p < ROWS / 2; ++p) o[p] *= __shfl(old, (2 * p + half) * 8, kWave);
      for (int e = 0; e < n; e += 2) {
        vec_t v[2][ROWS / 2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int p = 0; p < ROWS / 2; ++p) {  // (past the last: once more the last, with weight 0)
            const int r = min(r0 + 2 * p + half, rows - 1), rb = r / BQ;
            v[u][p] = *reinterpret_cast<const vec_t*>(record(base + min(e + u, n - 1), rb) + (r - rb * BQ) * D + at * PER);
          }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int p = 0; p < ROWS / 2; ++p) {
            const float z = __shfl(f, (2 * p + half) * 8 + ((e + u) & 7), kWave);
            o[p] += v[u][p] * (e + u < n ? z : 0.f);
          }
      }
    }
#pragma unroll
    for (int s = 1; s < 8; s <<= 1) L += __shfl_xor(L, s, kWave);
    const float inv = tree_inv(L);
#pragma unroll
    for (int p = 0; p < ROWS / 2; ++p) {
      const float z = __shfl(inv, (2 * p + half) * 8, kWave);
      const int r = r0 + 2 * p + half;
      if (r < rows) {
        T* op = out_at(r);
        if constexpr (PER == 4) {
          const float y[4] = {o[p][0] * z, o[p][1] * z, o[p][2] * z, o[p][3] * z};
          store4(op, y);
        } else {
#pragma unroll
          for (int c = 0; c < PER; ++c) stf(op + c, o[p][c] * z);
        }
      }
    }
  }
}

// One workgroup a sequence, thread i node i: ancestors by walking up.  A parent outside [0, i) is none.
__global__ __launch_bounds__(kMaxNodes) void k_tree_plan(int N, int W, const int32_t* __restrict__ parents,
                                                         const int32_t* __restrict__ pos0, const int32_t* __restrict__ len, int max_pos,
                                                         uint32_t* __restrict__ mask, int32_t* __restrict__ positions) {
  __shared__ int32_t par[kMaxNodes];
  const int b = blockIdx.x, i = threadIdx.x;
  const int64_t row = (int64_t)b * N + i, rows = (int64_t)gridDim.x * N;
  if (i < N) par[i] = parents ? parents[row] : i - 1;
  __syncthreads();
  if (i >= N) return;
  uint32_t words[kMaxNodes / 32] = {};
  int depth = -1;
  for (int at = i, up; at >= 0; at = up) {
#pragma unroll
    for (int w = 0; w < kMaxNodes / 32; ++w)
      if (at >> 5 == w) words[w] |= 1u << (at & 31);
    ++depth;
    up = par[at];
    if (up >= at) up = -1;
  }
#pragma unroll
  for (int w = 0; w < kMaxNodes / 32; ++w)
    if (w < W) mask[row * W + w] = words[w];
  const int64_t p = (int64_t)(pos0 ? pos0[b] : len[b]) + depth;
  const int pos = (int)(p < 0 ? 0 : p >= max_pos ? max_pos - 1 : p);
  positions[row] = pos;
  positions[rows + row] = pos;
  positions[2 * rows + row] = pos;
}

// How a launch runs: rows of a block (QW groups of 32 a wave), row blocks, shares of the tiles (a share:
// one workgroup per kv head and row block), the least tiles of one, and how much longer chunks may be.
// Measured, main kernel + merge in us (4 kv heads of 128 but for fp32):
//   stream or blocks of 128 rows: 64 sequences of one token over 8192 keys 192 + 5 or 225 + 7, 16 of 4 tokens
//   over 4000 29.6 + 4.7 or 31.4 + 5.0, 16 of 9 tokens (63 rows) 34.5 + 5.7 or 33.3 + 6.3.
//   32 or 64 rows a wave, 7 rows: 192 or 201 as above, 8 sequences of 300 to 1000 keys 13.4 or 16.1.
//   Shares: twice as many make the 16 of 4 tokens 38.0, 112 rows of 32 mixed trees 81 + 13 instead of 71 + 8.
//   Least tiles: one sequence of 4000 keys, 1, 3, 6, 12 tiles: 11.1 + 6.5, 10.7 + 5.1, 12.1 + 4.3, 13.4 + 3.8; 4
//   trees of 224 rows over 500 to 900 keys, 1, 4, 8, 16: 16.6 + 6.7, 16.1 + 5.3, 18.7 + 5.3, 24.2 + 4.8; fp32, 6
//   trees over 300 keys, 1, 4, 8: 10.2, 13.4, 17.0.
//   Slack: a third of it makes the 32 mixed trees 74.6 + 9.6, three times as much changes nothing.
struct TreePlan {
  bool stream;
  int QW, BQ, RB, shares, least, slack;
};
static TreePlan tree_plan(rp_dtype dt, int32_t N, int32_t Hq, int32_t Hkv) {
  TreePlan p;
  const int rows = N * (Hq / Hkv);
  p.stream = dt != RP_F32 && rows <= 64;
  p.QW = p.stream ? (rows + 31) / 32 : 1;
  p.BQ = dt == RP_F32 ? 32 : p.stream ? 32 * p.QW : 128;
  p.RB = (rows + p.BQ - 1) / p.BQ;
  // a stream workgroup has a CU's LDS to itself, of the others two share one
  p.shares = (p.stream ? 256 : 512) / (Hkv * p.RB);
  if (p.shares < 1) p.shares = 1;
  p.least = dt == RP_F32 ? 1 : p.stream ? 3 : 4;
  p.slack = p.stream ? 24 : 8;
  return p;
}

static size_t tree_records(const TreePlan& p, int32_t Hkv, int32_t D) {
  return (size_t)p.shares * 2 * Hkv * p.RB * tree_record(p.BQ, D);
}
size_t tree_partial_floats(rp_dtype dt, int32_t B, int32_t N, int32_t Hq, int32_t Hkv, int32_t D) {
  return tree_records(tree_plan(dt, N, Hq, Hkv), Hkv, D) + 2 * (size_t)B;
}

hipError_t launch_tree_attention(hipStream_t s, rp_dtype dt, const TreeArgs& args) {
  TreeArgs a = args;
  a.few = a.B <= 64 && (int64_t)a.B * (((int64_t)a.table_ld << a.lg) / 32 + kMaxNodes) < (int64_t)1 << 31;
  const TreePlan p = tree_plan(dt, a.N, a.Hq, a.Hkv);
  a.held = reinterpret_cast<int2*>(a.part + tree_records(p, a.Hkv, a.D));
  typedef std::integral_constant<int, 128> D128;
  typedef std::integral_constant<int, 64> D64;
  // up to four rows a wave slot of the chip: a wave a row (k_tree_merge has both measured)
  const int rows = a.N * (a.Hq / a.Hkv), per = (int64_t)rows * a.Hkv * a.B <= 4096 ? 1 : TM_MANY;
  const int64_t merge = (int64_t)((rows + TM_WAVES * per - 1) / (TM_WAVES * per)) * a.Hkv * a.B;
  auto join = [&](auto t_, auto d_) {
    typedef decltype(t_) T;
    constexpr int D = decltype(d_)::value;
    if (per == 1)
      k_tree_merge<T, D, 1><<<merge, 64 * TM_WAVES, 0, s>>>(a, p.BQ, p.RB);
    else
      k_tree_merge<T, D, TM_MANY><<<merge, 64 * TM_WAVES, 0, s>>>(a, p.BQ, p.RB);
  };
  if (dt == RP_F32) {
    const int grid = p.shares * a.Hkv * p.RB;
    if (a.D == 128) {
      k_tree_f32<128, 4><<<grid, 256, 0, s>>>(a, p.shares, p.least, p.slack, p.RB);
      join(float(), D128{});
    } else {
      k_tree_f32<64, 8><<<grid, 512, 0, s>>>(a, p.shares, p.least, p.slack, p.RB);
      join(float(), D64{});
    }
    return hipGetLastError();
  }
  with_half16(dt, [&](auto tag_) {
    using T = decltype(tag_);
    auto run = [&](auto d_) {
      constexpr int D = decltype(d_)::value;
      if (p.stream) {
        const int grid = p.shares * a.Hkv;
        // pages of 8 or 16 tokens: a tile in groups of 8 keys, each from its own page (as many buffer
        // resources again: the 64 sequences of 8192 keys 198 us instead of 193)
        const bool small = a.lg < 5;
        if (p.QW == 1)
          small ? k_tree_stream32<T, D, true><<<grid, 64 * TS_WAVES, 0, s>>>(a, p.shares, p.least, p.slack)
                : k_tree_stream32<T, D, false><<<grid, 64 * TS_WAVES, 0, s>>>(a, p.shares, p.least, p.slack);
        else
          small ? k_tree_stream64<T, D, true><<<grid, 64 * TS_WAVES, 0, s>>>(a, p.shares, p.least, p.slack)
                : k_tree_stream64<T, D, false><<<grid, 64 * TS_WAVES, 0, s>>>(a, p.shares, p.least, p.slack);
        join(T(), d_);
      } else {
        const int grid = (p.shares * a.Hkv + 7) / 8 * 8 * p.RB;
        k_tree_block<T, D><<<grid, 256, 0, s>>>(a, p.shares, p.least, p.slack, p.RB);
        join(T(), d_);
      }
    };
    if (a.D == 128)
      run(D128{});
    else
      run(D64{});
  });
  return hipGetLastError();
}

hipError_t launch_tree_plan(hipStream_t s, int32_t B, int32_t N, int32_t W, const int32_t* parents, const int32_t* pos0,
                            const int32_t* len, int32_t max_pos, uint32_t* mask, int32_t* positions) {
  k_tree_plan<<<B, kMaxNodes, 0, s>>>(N, W, parents, pos0, len, max_pos, mask, positions);
  return hipGetLastError();
}

}  // namespace rp
