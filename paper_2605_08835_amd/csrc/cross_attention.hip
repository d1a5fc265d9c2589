// Attention of each row's queries over a text of its own length:
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q . k_j)
// over the keys of the row's context that take part.
//
// A "row" below is one (query, head) pair of a K/V head: with rep heads to a
// K/V head, row r of an image and K/V head g is query r / rep, head g rep +
// r % rep, so shared heads fill the tiles like further queries.
//
//  * Many rows (bf16): flash attention on MFMA.  A wave owns 32 rows, the
//    block shares tiles of 64 keys in LDS.  Scores are computed transposed,
//    S^T = K Q^T, so that a lane holds one row's scores: its maximum and
//    rescale are per-lane, and P^T feeds O^T = V^T P^T from the registers.
//    V lies in LDS as it came (key by key); the transposing LDS read hands
//    each lane four keys of one channel.
//  * fp32: the same on fp32 MFMAs.
//  * Few rows (at most 128): bound by the bytes of K and V.  The waves of a
//    block share out the keys of one tile of 32 rows and meet only at the end.
//    fp32 with at most 8 rows needs no tile: lanes share a key's channels, and
//    every lane group runs an online softmax of its own.
//  * Few rows over long texts are split along the keys into ranges of a fixed
//    length, whose unnormalised results a second kernel joins in order.  The
//    ranges start at the text's own first key: a row's bits depend neither on
//    the batch nor on the longest text in it.
// Keys that take no part are never read (their memory may hold NaN): masks
// become a bit per key of a tile before its loads are issued.
#include <type_traits>

#include "device_common.h"
#include "kernels.h"

namespace sd {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float TAU = 8.0f;  // the running maximum moves when a tile's passes it by this much (log2 units)

// What image `img` reads: its context's first key (elements of K and V, mask byte) and the count.
struct Text {
  long k0, v0, m0;
  int len;
};
__device__ __forceinline__ Text text_of(const CrossArgs& a, int img) {
  Text t = {0, 0, 0, 0};
  const int c = a.kv_index ? a.kv_index[img] : img;
  if (c < 0 || c >= a.n_ctx) return t;
  int len = a.kv_len ? a.kv_len[c] : a.max_len;
  len = min(max(len, 0), a.max_len);
  if (a.kv_start) {
    const long start = a.kv_start[c];
    if (start < 0 || start >= a.kv_tokens) return t;
    len = (int)min((long)len, a.kv_tokens - start);
    t.k0 = start * a.k_ld;
    t.v0 = start * a.v_ld;
    t.m0 = start;
  } else {
    t.k0 = (long)c * a.k_ctx;
    t.v0 = (long)c * a.v_ctx;
    t.m0 = (long)c * a.max_len;
  }
  t.len = len;
  return t;
}

// Block -> (K/V head, row tile, split, image).  Consecutive blocks go to the 8
// XCDs in turn, each with an L2 of its own.
//  * together > 0: the row tiles of one K/V head read the same keys, so the tiles
//    of `together` neighbouring heads stay on one XCD, next to each other in time (over
//    all 8, K and V came from memory 8 times).
//  * together = 0, where keys are read once or are few: all K/V heads of one
//    tile stay on one XCD, since their rows share cache lines of q, o, K and V
//    (48 x 4096 rows, 8 heads of 40, up to 77 keys: 97 us against 121 over all XCDs).
struct Place {
  int g, tile, split, img;
  bool on;
};
__device__ __forceinline__ Place place_of(int kv_heads, int tiles, int splits, int n, int together) {
  const unsigned id = blockIdx.x, xcd = id & 7, i = id >> 3;
  Place p;
  if (together) {
    const unsigned per = (unsigned)tiles * splits * together, groups = kv_heads / together;
    const unsigned u = i / per * 8 + xcd, t = i % per;
    p.on = u < groups * n;
    p.g = u % groups * together + t % together;
    p.img = u / groups;
    p.tile = t / together % tiles;
    p.split = t / together / tiles;
  } else {
    const unsigned t = i / kv_heads * 8 + xcd;
    p.g = i % kv_heads;
    p.on = t < (unsigned)tiles * splits * n;
    p.tile = t % tiles;
    p.split = t / tiles % splits;
    p.img = t / tiles / splits;
  }
  return p;
}
static unsigned place_blocks(long kv_heads, long tiles, long splits, long n, long together) {
  if (!together) return (unsigned)((tiles * splits * n + 7) / 8 * 8 * kv_heads);
  return (unsigned)((kv_heads / together * n + 7) / 8 * 8 * tiles * splits * together);
}
// Heads whose rows fill whole lines of 128 bytes, where that many divide the
// heads and leave every XCD two of them (16 x 4096 rows, 8 heads of 40, up to 300
// keys: 67 us against 77 one by one); else one; none where that left over a
// quarter of the XCDs' turns empty.
static int place_together(const CrossArgs& a, int el) {
  int h = 1;
  while (h * a.d * el % 128) h *= 2;
  if (a.kv_heads % h || (long)a.n * (a.kv_heads / h) < 16) h = 1;
  const long groups = (long)a.n * (a.kv_heads / h), rounds = (groups + 7) / 8;
  return groups * 4 >= rounds * 24 ? h : 0;
}

// The kernel of a call, by the rows of a K/V head, and its ranges of `keys` (0:
// not split): kind 0 up to 8 rows, 1 up to 128, 2 past that.  The ranges cannot
// follow the number of images or the longest text (a row's bits), so each is a
// compromise between calls that fill the card and calls that do not (us; n x
// queries, heads of 64 over so many keys):
//   up to 128 rows 1024 keys (in brackets 512, 2048): 4 x 1, 20 heads, 9000 to
//   16384 64 (63, 68); 1 x 16, 8 heads, 4000 to 8000 16 (13, 23); 32 x 40, 8
//   heads, 300 to 700 15 (28, 14);
//   up to 512 rows 512 keys (1024, not split): 1 x 200, 8 heads, 4000 to 8000 22
//   (29, 144); 8 x 512, 20 heads, 600 to 1100 95 (96, 44);
//   past that not split (512 keys): 16 x 1024, 20 heads, 600 to 1100 126 (337);
//   1 x 1024, 8 heads, 16000 285 (79).
struct Plan {
  int kind, keys, splits;
};
static Plan plan_of(int rep, int n_q, int max_len) {
  const long rows = (long)rep * n_q;
  Plan p;
  p.kind = rows <= 8 ? 0 : rows <= 128 ? 1 : 2;
  p.keys = p.kind <= 1 ? 1024 : rows <= 512 ? 512 : 0;
  p.splits = p.keys && max_len > p.keys ? (max_len + p.keys - 1) / p.keys : 1;
  return p;
}

// Scratch of a split call: per (image, K/V head, row, split) d floats of
// sum p v, then behind all of them (m, l): p = exp2(score - m), l = sum p.
struct Scratch {
  float *o, *ml;
};
__device__ __forceinline__ Scratch scratch_at(const CrossArgs& a, int img, int g, int row, int split, int splits) {
  const long rows = (long)a.rep * a.n_q, at = (((long)img * a.kv_heads + g) * rows + row) * splits + split;
  return {a.scratch + at * a.d, a.scratch + (long)a.n * a.kv_heads * rows * splits * a.d + 2 * at};
}

// Row r of a K/V head: its query, and its head among the rep that share.
struct RowAt {
  int t, h;
};
__device__ __forceinline__ RowAt row_at(const CrossArgs& a, int r) {
  if (a.rep == 1) return {r, 0};
  const int t = (int)(__umulhi((unsigned)r, a.rep_mul) >> a.rep_shift);
  return {t, r - t * a.rep};
}

// What a row's exponents are taken against: its running maximum, or 0 as long as
// every key so far scored -inf (then every p is 0; -inf minus -inf is NaN).
__device__ __forceinline__ float exp_ref(float m) { return m == -INFINITY ? 0.f : m; }

__device__ __forceinline__ float2 half_swap(float v) {  // (v of lanes l and l ^ 32)
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
#else
  return make_float2(v, v);
#endif
}

}  // namespace

// ------------------------------------------------------------------ few rows, fp32
// RB rows (a power of two) per K/V head.  LPK lanes (a power of two) hold a key's
// channels, 8 each; a wave has 64 / LPK key groups, U keys of each in flight.
template <int RB, int LPK>
__global__ __launch_bounds__(512) void cross_few_kernel(CrossArgs a, int keys, int splits) {
  constexpr int U = RB <= 2 ? 4 : 2, NG = 64 / LPK, NW = 8, STEP = NW * NG * U;
  const Place p = place_of(a.kv_heads, 1, splits, a.n, 0);
  if (!p.on) return;
  const Text tx = text_of(a, p.img);
  const int k_begin = p.split * keys, k_end = splits > 1 ? min(tx.len, k_begin + keys) : tx.len;
  if (splits > 1 && k_begin >= tx.len) return;  // (the join knows the text's length)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, ch = (lane % LPK) * 8, grp = lane / LPK;
  const int rows = a.rep * a.n_q;
  const bool has = ch < a.d;
  const float* K = (const float*)a.k + tx.k0 + p.g * a.k_head + ch;
  const float* V = (const float*)a.v + tx.v0 + p.g * a.v_head + ch;
  const uint8_t* mask = a.mask ? a.mask + tx.m0 : nullptr;

  float q[RB][8], o[RB][8], m[RB], l[RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
#pragma unroll
    for (int e = 0; e < 8; ++e) q[r][e] = o[r][e] = 0.f;
    m[r] = -INFINITY;
    l[r] = 0.f;
    if (r < rows && has) {
      const int t = r / a.rep, h = p.g * a.rep + r % a.rep;
      load8f((const float*)a.q + (long)p.img * a.q_img + t * a.q_ld + h * a.q_head + ch, q[r]);
#pragma unroll
      for (int e = 0; e < 8; ++e) q[r][e] *= a.scale * LOG2E;
    }
  }
  // key u of this lane group in the step from k on
  auto key_of = [&](int k, int u) { return k + (u * NW + wave) * NG + grp; };
  auto part = [&](int key) { return key < k_end && (!mask || mask[key]); };
  bool on[U];
#pragma unroll
  for (int u = 0; u < U; ++u) on[u] = part(key_of(k_begin, u));
  for (int k = k_begin; k < k_end; k += STEP) {
    float kf[U][8], vf[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int e = 0; e < 8; ++e) kf[u][e] = vf[u][e] = 0.f;
      const long key = key_of(k, u);
      if (on[u] && has) {
        load8f(K + key * a.k_ld, kf[u]);
        load8f(V + key * a.v_ld, vf[u]);
      }
    }
    bool next[U];
#pragma unroll
    for (int u = 0; u < U; ++u) next[u] = part(key_of(k + STEP, u));
    float s[RB][U];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < RB; ++r) {
        float d = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) d = fmaf(q[r][e], kf[u][e], d);
#pragma unroll
        for (int x = 1; x < LPK; x <<= 1) d += __shfl_xor(d, x, 64);
        s[r][u] = on[u] ? d : -INFINITY;
      }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
      float mn = m[r];
#pragma unroll
      for (int u = 0; u < U; ++u) mn = fmaxf(mn, s[r][u]);
      const float ref = exp_ref(mn);
      const float al = __builtin_amdgcn_exp2f(m[r] - ref);
      m[r] = mn;
      l[r] *= al;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[r][e] *= al;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float pr = __builtin_amdgcn_exp2f(s[r][u] - ref);
        l[r] += pr;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[r][e] = fmaf(pr, vf[u][e], o[r][e]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) on[u] = next[u];
  }
  // Join the key groups of the wave, then the waves through LDS, in order.
  __shared__ float so[NW][RB][LPK * 8], sm[NW][RB], sl[NW][RB];
#pragma unroll
  for (int r = 0; r < RB; ++r) {
    float mw = m[r];
#pragma unroll
    for (int x = LPK; x < 64; x <<= 1) mw = fmaxf(mw, __shfl_xor(mw, x, 64));
    const float f = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[r] - mw);
    float lw = l[r] * f;
#pragma unroll
    for (int x = LPK; x < 64; x <<= 1) lw += __shfl_xor(lw, x, 64);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float v = o[r][e] * f;
#pragma unroll
      for (int x = LPK; x < 64; x <<= 1) v += __shfl_xor(v, x, 64);
      if (grp == 0) so[wave][r][ch + e] = v;
    }
    if (lane == 0) {
      sm[wave][r] = mw;
      sl[wave][r] = lw;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < rows * a.d; i += 64 * NW) {
    const int r = i / a.d, c = i - r * a.d;
    float mt = sm[0][r];
#pragma unroll
    for (int w = 1; w < NW; ++w) mt = fmaxf(mt, sm[w][r]);
    float v = 0.f, lt = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = sm[w][r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[w][r] - mt);
      v = fmaf(f, so[w][r][c], v);
      lt = fmaf(f, sl[w][r], lt);
    }
    if (splits > 1) {
      const Scratch sc = scratch_at(a, p.img, p.g, r, p.split, splits);
      sc.o[c] = v;
      if (c == 0) {
        sc.ml[0] = mt;
        sc.ml[1] = lt;
      }
    } else {
      const int t = r / a.rep, h = p.g * a.rep + r % a.rep;
      ((float*)a.o)[(long)p.img * a.o_img + t * a.o_ld + h * a.o_head + c] = lt == 0.f ? 0.f : v * (1.0f / lt);
    }
  }
}

// ------------------------------------------------------------------ join
// One wave per row, one block per wave: the splits of its text in order.  Lane
// u holds (m, l) of split u, lanes hold a channel of every 64; the loads of U
// splits are in flight at once (80 rows of 64, 9 to 16 splits: 4.7 us, one split
// after another 12.9).
template <typename T, int NI>
__global__ __launch_bounds__(64) void cross_join_kernel(CrossArgs a, int keys, int splits) {
  constexpr int U = NI == 1 ? 16 : 8;
  const int lane = threadIdx.x;
  const unsigned rows = (unsigned)(a.rep * a.n_q), e = blockIdx.x;
  const int r = (int)(e % rows), g = (int)(e / rows % a.kv_heads), img = (int)(e / rows / a.kv_heads);
  const int ns = (text_of(a, img).len + keys - 1) / keys;
  const Scratch sc = scratch_at(a, img, g, r, 0, splits);
  float m = -INFINITY, l = 0.f;
  if (lane < ns) m = sc.ml[2 * lane], l = sc.ml[2 * lane + 1];
  float mt = m;
  for (int s = lane + 64; s < ns; s += 64) mt = fmaxf(mt, sc.ml[2 * s]);
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) mt = fmaxf(mt, __shfl_xor(mt, x, 64));
  float v[NI], lt = 0.f;
#pragma unroll
  for (int i = 0; i < NI; ++i) v[i] = 0.f;
  for (int s0 = 0; s0 < ns; s0 += 64) {
    if (s0) {
      m = -INFINITY, l = 0.f;
      if (s0 + lane < ns) m = sc.ml[2 * (s0 + lane)], l = sc.ml[2 * (s0 + lane) + 1];
    }
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mt);
    for (int u0 = s0; u0 < min(s0 + 64, ns); u0 += U) {
      float x[U][NI];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          x[u][i] = 0.f;
          if (u0 + u < ns && lane + 64 * i < a.d) x[u][i] = sc.o[(long)(u0 + u) * a.d + lane + 64 * i];
        }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float fu = __shfl(f, u0 - s0 + u, 64);
        lt = fmaf(fu, __shfl(l, u0 - s0 + u, 64), lt);
#pragma unroll
        for (int i = 0; i < NI; ++i) v[i] = fmaf(fu, x[u][i], v[i]);
      }
    }
  }
  const float inv = lt == 0.f ? 0.f : 1.0f / lt;
  T* o = (T*)a.o + (long)img * a.o_img + (r / a.rep) * a.o_ld + (g * a.rep + r % a.rep) * a.o_head;
#pragma unroll
  for (int i = 0; i < NI; ++i)
    if (lane + 64 * i < a.d) o[lane + 64 * i] = from_f<T>(v[i] * inv);
}
template <typename T>
static void launch_join(const CrossArgs& a, const Plan& p, hipStream_t s) {
  const unsigned grid = (unsigned)((long)a.n * a.kv_heads * a.rep * a.n_q);
  if (a.d <= 64) cross_join_kernel<T, 1><<<grid, 64, 0, s>>>(a, p.keys, p.splits);
  else if (a.d <= 128) cross_join_kernel<T, 2><<<grid, 64, 0, s>>>(a, p.keys, p.splits);
  else cross_join_kernel<T, 4><<<grid, 64, 0, s>>>(a, p.keys, p.splits);
}

// ------------------------------------------------------------------ many rows, bf16
namespace {

constexpr int KT = 64;  // keys per tile

// LDS row of V: a multiple of 16 channels whose four rows a transposing read
// takes lie in different banks (an odd number of 32-byte units, or a row that
// fills a multiple of 64 but not of 128 or 256 bytes).
__host__ __device__ constexpr int v_row(int d16) { return d16 * 2 % 128 == 0 ? d16 + 16 : d16; }

// Four keys (LDS rows) of one channel for each lane of a group of 16: lane i
// names the 8 bytes of row i / 4, channels 4 (i % 4) on, and gets channel i of rows 0 to 3.
__device__ __forceinline__ bf16x4 read_transposed(const bf16* p) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
#else
  return *(const bf16x4*)p;
#endif
}

// l + the eight rounded probabilities, two to an instruction (taking them apart
// again cost three each, a third of a 64-key tile's vector instructions).
__device__ __forceinline__ float sum_probs(bf16x8 p, float l) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 one = {(bf16)1.0f, (bf16)1.0f};
  l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 0, 1), one, l, false);
  l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 2, 3), one, l, false);
  l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 4, 5), one, l, false);
  l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p, p, 6, 7), one, l, false);
#endif
  return l;
}

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}

}  // namespace

// D16: head width rounded up to a width the kernel is built for.  SF: d < D16,
// so that channel d of V in LDS is free: it holds ones, and row d of O^T
// becomes the sum of the (rounded) probabilities.  Four waves of 32 rows.
// SHORT: no text is longer than the two tiles that LDS holds; they are staged
// once, and the waves pass `passes` groups of rows each over them without
// meeting again (48 x 4096 rows, 8 heads of 40, up to 77 keys: 91 us, staging
// them for every 128 rows 149).  Its arithmetic on a row is the same.  What
// bounds it is memory: 80-byte rows of a 640-byte token reach 3.3 TB/s with the
// arithmetic left out, which alone takes 47 us; three waves per SIMD hide part
// of one behind the other.
// Otherwise a wave's order of work on a tile bounds it, which only other waves
// overlap: score products, maximum, exponentials, value products (vector ALU
// busy 54 % of the time, the matrix unit 27 %): 16 x 1024 rows, 20 heads of 64,
// padded texts of 200 to 512 keys 59 us, 430 TFLOP/s.
// Two waves per SIMD up to 128 channels, though a few registers spill there (8 x
// 2048 rows, 8 heads of 128, up to 512 keys: 61 us against 66).
template <int D16, bool SF, bool SHORT>
__global__ __launch_bounds__(256, D16 <= 48 || (D16 == 64 && !SHORT) ? 3 : D16 <= 128 ? 2 : 1) void cross_bf16_kernel(
    CrossArgs a, int keys, int tiles, int splits, int passes, int together) {
  constexpr int NW = 4, NJ = D16 / 16, ND = (D16 + 31) / 32, NT = 64 * NW, LDK = D16 + 8, LDV = v_row(D16);
  // A tile is moved by passes of NT / LPR keys, LPR lanes (a power of two) a key
  constexpr int LPR = D16 <= 32 ? 4 : D16 <= 64 ? 8 : D16 <= 128 ? 16 : 32, RPP = NT / LPR < KT ? NT / LPR : KT, CPT = KT / RPP;
  __shared__ __attribute__((aligned(16))) bf16 Ks[2][KT * LDK];
  __shared__ __attribute__((aligned(16))) bf16 Vs[2][KT * LDV + 32];  // (the last rows are read past their end where D16 % 32)
  __shared__ __attribute__((aligned(16))) bf16 Os[SHORT ? NW * 32 * LDK : 8];
  const Place p = place_of(a.kv_heads, tiles, splits, a.n, SHORT ? 0 : together);
  if (!p.on) return;
  const Text tx = text_of(a, p.img);
  const int k_begin = p.split * keys, k_end = splits > 1 ? min(tx.len, k_begin + keys) : tx.len;
  if (splits > 1 && k_begin >= tx.len) return;  // (the join knows the text's length)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lq = lane & 31, lh = lane >> 5;
  const int rows = a.rep * a.n_q, d = a.d;
  int r0 = (p.tile * passes * NW + wave) * 32;  // (uniform)
  const uint8_t* mask = a.mask ? a.mask + tx.m0 : nullptr;
  // (a scale of 0 or below: uniform weights, or -q, under a positive one)
  const float sl2 = a.scale == 0.f ? LOG2E : fabsf(a.scale) * LOG2E;
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;

  // Q^T fragments (B operand): row rg + lq, channels 16 j + 8 lh + [0, 8)
  auto load_q = [&](int rg, bf16x8 (&qf)[NJ]) __attribute__((always_inline)) {
    uint4 v[NJ];
    const int n = a.scale == 0.f ? 0 : min(32, rows - rg);
    if (a.rep == 1) {  // (32 rows from one address on; what lies past them, and channels from d on, read as zero)
      const bf16* Q = (const bf16*)a.q + (long)p.img * a.q_img + (long)rg * a.q_ld + p.g * a.q_head;
      const __amdgpu_buffer_rsrc_t qr = make_rsrc(Q, n <= 0 ? 0 : ((n - 1) * (long)a.q_ld + d) * 2);
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        v[j] = __builtin_bit_cast(uint4, buf_load16(qr, 16 * j + 8 * lh < d ? (lq * (int)a.q_ld + 16 * j + 8 * lh) * 2 : OOB));
    } else {
      const RowAt at = row_at(a, rg + lq);
      const bf16* Q = (const bf16*)a.q + (long)p.img * a.q_img + at.t * a.q_ld + (p.g * a.rep + at.h) * a.q_head;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        v[j] = make_uint4(0, 0, 0, 0);
        if (lq < n && 16 * j + 8 * lh < d) v[j] = *(const uint4*)(Q + 16 * j + 8 * lh);
      }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      v[j].x ^= flip;
      v[j].y ^= flip;
      v[j].z ^= flip;
      v[j].w ^= flip;
      qf[j] = __builtin_bit_cast(bf16x8, v[j]);
    }
  };
  bf16x8 qf[NJ];
  load_q(r0, qf);
  if constexpr (SF)  // ones in channel d of every key of both buffers
    for (int i = tid; i < 2 * KT; i += NT) {
      bf16x8 v = {};
      v[0] = (bf16)1.0f;
      *(bf16x8*)&Vs[i / KT][(i % KT) * LDV + d] = v;
    }
  f32x16 o[ND];  // (set by the first tile that holds a key)
  float m_run, l_run;
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
    m_run = -INFINITY;
    l_run = 0.f;
  };

  // A thread's pieces of a tile: keys pk + RPP i, channels pc on.  (Offsets past a
  // resource's end, as those of channels from d on and of keys that take no part, read as zero.)
  const int pk = tid / LPR, pc = tid % LPR * 8;
  const bool mine = pk < RPP && pc < D16;  // (fewer than NT threads where LPR is wide or the tile short)
  const int ko = pc < d ? (pk * (int)a.k_ld + pc) * 2 : OOB, vo = pc < d ? (pk * (int)a.v_ld + pc) * 2 : OOB;
  const bf16* K = (const bf16*)a.k + tx.k0 + p.g * a.k_head;
  const bf16* V = (const bf16*)a.v + tx.v0 + p.g * a.v_head;
  bf16x8 rk[CPT], rv[CPT];
  auto fetch = [&](int k0, uint64_t bits) __attribute__((always_inline)) {
    const int n = min(KT, k_end - k0);
    const __amdgpu_buffer_rsrc_t kr = make_rsrc(K + (long)k0 * a.k_ld, ((n - 1) * (long)a.k_ld + d) * 2);
    const __amdgpu_buffer_rsrc_t vr = make_rsrc(V + (long)k0 * a.v_ld, ((n - 1) * (long)a.v_ld + d) * 2);
    const uint64_t b = bits >> (pk & 63);
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const bool on = (b >> (RPP * i & 63)) & 1;
      rk[i] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(kr, on ? ko + i * RPP * (int)a.k_ld * 2 : OOB, 0, 0));
      rv[i] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(vr, on ? vo + i * RPP * (int)a.v_ld * 2 : OOB, 0, 0));
    }
  };
  auto stage = [&](int b) __attribute__((always_inline)) {
    if (mine)
#pragma unroll
      for (int i = 0; i < CPT; ++i) {
        *(bf16x8*)&Ks[b][(pk + RPP * i) * LDK + pc] = rk[i];
        if (!SF || pc < d) *(bf16x8*)&Vs[b][(pk + RPP * i) * LDV + pc] = rv[i];
      }
  };
  // which of the 64 keys from k0 on take part: lane's own, as loaded; then a bit per key
  auto own_key = [&](int k0) -> bool {
    const int k = k0 + lane;
    return k < k_end && (!mask || mask[k]);
  };

  bf16x8 ones = {};  // B operand of the masks: ones for k = 0
  if (lh == 0) ones[0] = (bf16)1.0f;

  // NKT: 32-key halves of the tile that hold keys at all.  FIRST: nothing has
  // been summed yet.
  auto tile = [&](auto nkt, auto first, int b, uint64_t bits) __attribute__((always_inline)) {
    constexpr int NKT = decltype(nkt)::value;
    constexpr bool FIRST = decltype(first)::value;
    const bf16 *Kb = Ks[b], *Vb = Vs[b];
    f32x16 s[NKT];
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt) {
      // Keys that take no part start from -inf: one product of a column of 0
      // or -inf per key with a row of ones (a select per score cost three
      // vector instructions each, and the vector ALU bounds this kernel).
      const f32x16 zero = {};
      bf16x8 off = {};
      if (lh == 0) off[0] = __builtin_bit_cast(bf16, (unsigned short)(bits >> (32 * kt + lq) & 1 ? 0 : 0xFF80));
      const f32x16 start = mfma32(off, ones, zero);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const bf16x8 kf = *(const bf16x8*)&Kb[(kt * 32 + lq) * LDK + 16 * j + 8 * lh];
        s[kt] = mfma32(kf, qf[j], j ? s[kt] : start);
      }
    }
    // register r of half kt: key 32 kt + 8 (r / 4) + 4 lh + r % 4
    float v = s[0][0];
#pragma unroll
    for (int kt = 0; kt < NKT; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) v = fmaxf(v, s[kt][r]);
    const float2 h = half_swap(v);
    const float mt = fmaxf(h.x, h.y) * sl2;
    const bool need = FIRST || mt > m_run + TAU;
    if constexpr (FIRST) m_run = mt;
    if (!FIRST && __any(need)) {  // (where a row's maximum stays, its sums are multiplied by one)
      const float al = need ? __builtin_amdgcn_exp2f(m_run - mt) : 1.0f;
      m_run = need ? mt : m_run;
      l_run *= al;
#pragma unroll
      for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] *= al;
    }
    const float ref = exp_ref(m_run);
    // O^T += V^T P^T, 16 keys at a time: slot (lh, i) of slice u is key 16 u +
    // 8 (i / 4) + 4 lh + i % 4, register 8 (u % 2) + i of half u / 2.  The
    // probabilities are rounded to bf16 (by up to 2^-8 of each, half a step) and
    // summed as rounded, so that the rounding cancels where one key prevails.
    // Against 64 bits a result is 0.0022 off in the mean then (16 x 1024 rows
    // over 200 to 512 keys), 0.0017 with fp32 probabilities, where only the result
    // is rounded.  Keeping the rest as a second part, as for few rows, takes 82 us in
    // place of 59 there, and 104 in place of 91 for 48 x 4096 rows over up to 77 keys.
#pragma unroll
    for (int u = 0; u < 2 * NKT; ++u) {
      bf16x8 vf[ND];
#pragma unroll
      for (int t = 0; t < ND; ++t) {
        const bf16* at = &Vb[(16 * u + 4 * lh + ((lane & 15) >> 2)) * LDV + t * 32 + (lane & 16) + 4 * (lane & 3)];
        const bf16x4 lo = read_transposed(at), hi = read_transposed(at + 8 * LDV);
        vf[t] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
      bf16x8 pf;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        pf[i] = (bf16)__builtin_amdgcn_exp2f(fmaf(s[u >> 1][8 * (u & 1) + i], sl2, -ref));
      if constexpr (!SF) l_run = sum_probs(pf, FIRST && u == 0 ? 0.f : l_run);
#pragma unroll
      for (int t = 0; t < ND; ++t) {
        const f32x16 zero = {};
        o[t] = mfma32(vf[t], pf, FIRST && u == 0 ? zero : o[t]);
      }
    }
  };
  bool any_key = false;  // (uniform)
  auto tile_of = [&](auto first, int b, uint64_t bits) __attribute__((always_inline)) {
    if (bits >> 32)
      tile(std::integral_constant<int, 2>{}, first, b, bits);
    else if (bits)
      tile(std::integral_constant<int, 1>{}, first, b, bits);
    any_key = any_key || bits;
  };

  // O^T: lane holds channels 32 t + 8 (r / 4) + 4 lh + r % 4 of its row.
  auto finish = [&]() __attribute__((always_inline)) {
    if (!any_key) clear();
    float l = l_run;
    if constexpr (SF) {  // (d is a multiple of 8: register 0 of a quad of half 0)
#pragma unroll
      for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (32 * t + 8 * i == d) l = o[t][4 * i];
      l = lh == 0 ? l : 0.f;
    }
    const float2 h = half_swap(l);
    l = h.x + h.y;
    const int r = r0 + lq;
    if (!SHORT && splits > 1) {
      if (r < rows) {
        const Scratch sc = scratch_at(a, p.img, p.g, r, p.split, splits);
#pragma unroll
        for (int t = 0; t < ND; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int c = 32 * t + 8 * i + 4 * lh;
            if (c < d) *(float4*)(sc.o + c) = make_float4(o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]);
          }
        if (lh == 0) {
          sc.ml[0] = m_run;
          sc.ml[1] = l;
        }
      }
      return;
    }
    // Rows are laid out in LDS (K's tiles are done with, unless SHORT) and leave 16 bytes a lane.
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    bf16* R = (SHORT ? Os : &Ks[0][0]) + wave * 32 * LDK;
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = 32 * t + 8 * i + 4 * lh;
        if (c < d) {
          bf16x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = (bf16)(o[t][4 * i + e] * inv);
          *(bf16x4*)(R + lq * LDK + c) = w;
        }
      }
    asm volatile("" ::: "memory");  // (one wave's LDS accesses complete in order)
    const int c = lane % LPR * 8, row0 = lane / LPR;
    bf16* O = (bf16*)a.o + (long)p.img * a.o_img + p.g * a.rep * a.o_head + c;
    if (c < d) {
      if (a.rep == 1) {
        O += (long)r0 * a.o_ld;
#pragma unroll
        for (int i = 0; i < 32; i += 64 / LPR)
          if (r0 + row0 + i < rows) *(bf16x8*)(O + (row0 + i) * (int)a.o_ld) = *(const bf16x8*)(R + (row0 + i) * LDK + c);
      } else {
#pragma unroll
        for (int i = 0; i < 32; i += 64 / LPR)
          if (r0 + row0 + i < rows) {
            const RowAt at = row_at(a, r0 + row0 + i);
            *(bf16x8*)(O + at.t * a.o_ld + at.h * a.o_head) = *(const bf16x8*)(R + (row0 + i) * LDK + c);
          }
      }
    }
    asm volatile("" ::: "memory");
  };

  if constexpr (SHORT) {
    const uint64_t b0 = __ballot(own_key(0)), b1 = __ballot(own_key(KT));
    if (k_end > 0) fetch(0, b0);
    stage(0);
    if (k_end > KT) {
      fetch(KT, b1);
      stage(1);
    }
    __syncthreads();
    for (int it = 0; it < passes; ++it) {
      bf16x8 qn[NJ];
      const int rn = r0 + NW * 32;
      if (it + 1 < passes && rn < rows) load_q(rn, qn);
      if (r0 < rows) {
        const int bf = b0 ? 0 : 1;  // (the first tile that holds a key)
        tile_of(std::true_type{}, bf, b0 ? b0 : b1);
        if (b0) tile_of(std::false_type{}, 1, b1);
        finish();
      }
      if (it + 1 < passes) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) qf[j] = qn[j];
        r0 = rn;
      }
    }
  } else {
    if (k_begin < k_end) {
      uint64_t bits = __ballot(own_key(k_begin));
      fetch(k_begin, bits);
      bool nk = own_key(k_begin + KT);
      stage(0);
      __syncthreads();
      for (int k0 = k_begin, b = 0; k0 < k_end; k0 += KT, b ^= 1) {
        uint64_t next = 0;
        const bool more = k0 + KT < k_end;
        if (more) {
          next = __ballot(nk);
          fetch(k0 + KT, next);
          nk = own_key(k0 + 2 * KT);
        }
        if (any_key)
          tile_of(std::false_type{}, b, bits);
        else
          tile_of(std::true_type{}, b, bits);
        if (more) stage(b ^ 1);
        __syncthreads();
        bits = next;
      }
    }
    finish();
  }
}

// ------------------------------------------------------------------ few rows, bf16
// The results of a block's waves (row by row in LDS, `area` floats apart), whose
// maxima and sums are sm and sl, joined in order: to the output, or as one split's
// result to scratch.  Four channels a thread.
template <typename T, int NW>
__device__ __forceinline__ void join_waves(const CrossArgs& a, const Place& p, int splits, int r0, int here, const float* res,
                                           int area, int ldo, const float (&sm)[NW][32], const float (&sl)[NW][32]) {
  const int d4 = a.d >> 2;
  for (int i = threadIdx.x; i < here * d4; i += 64 * NW) {
    const int row = i / d4, c = (i - row * d4) * 4;
    float mt = sm[0][row];
#pragma unroll
    for (int w = 1; w < NW; ++w) mt = fmaxf(mt, sm[w][row]);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    float lt = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float f = sm[w][row] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[w][row] - mt);
      const f32x4 x = *(const f32x4*)(res + w * area + row * ldo + c);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = fmaf(f, x[e], v[e]);
      lt = fmaf(f, sl[w][row], lt);
    }
    if (splits > 1) {
      const Scratch sc = scratch_at(a, p.img, p.g, r0 + row, p.split, splits);
      *(f32x4*)(sc.o + c) = v;
      if (c == 0) {
        sc.ml[0] = mt;
        sc.ml[1] = lt;
      }
    } else {
      const RowAt at = row_at(a, r0 + row);
      const float inv = lt == 0.f ? 0.f : 1.0f / lt;
      T* out = (T*)a.o + (long)p.img * a.o_img + at.t * a.o_ld + (p.g * a.rep + at.h) * a.o_head + c;
      if constexpr (std::is_same<T, float>::value) {
        *(f32x4*)out = v * inv;
      } else {
        bf16x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (bf16)(v[e] * inv);
        *(bf16x4*)out = w;
      }
    }
  }
}

// A block takes 32 rows and a range of keys; its waves share the keys out, 32 at
// a time, each with a piece of LDS, an online softmax and an O^T of its own,
// and are joined at the end.  No barrier until then: what bounds it is the
// bytes of K and V, so waves only have to keep loads in flight: 4.9 TB/s, one
// query over 9000 to 16384 keys, 4 x 20 heads of 64 in 57 us.  (The tile is
// mostly empty for one query; its products still take less time than the loads.)
template <int D16, bool SF, int NW>
__global__ __launch_bounds__(64 * NW, D16 <= 64 ? 3 : 1) void cross_keys_kernel(CrossArgs a, int keys, int tiles, int splits,
                                                                                  int together) {
  constexpr int NJ = D16 / 16, ND = (D16 + 31) / 32, LDK = D16 + 8, LDV = v_row(D16), KW = 32;
  constexpr int LPR = D16 <= 32 ? 4 : D16 <= 64 ? 8 : D16 <= 128 ? 16 : 32, RPP = 64 / LPR, CPT = KW / RPP;
  constexpr int WAVE = KW * LDK + KW * LDV + 32, LDO = D16 + 4;  // (bf16 of a wave's LDS; floats of a row of its result)
  static_assert(WAVE * 2 >= 32 * LDO * 4 || D16 > 160, "a wave's result takes the place of its tiles");
  constexpr int AREA = WAVE * 2 > 32 * LDO * 4 ? WAVE * 2 : 32 * LDO * 4;
  __shared__ __attribute__((aligned(16))) uint8_t smem[NW * AREA];
  __shared__ float sm[NW][32], sl[NW][32];
  const Place p = place_of(a.kv_heads, tiles, splits, a.n, together);
  if (!p.on) return;
  const Text tx = text_of(a, p.img);
  const int k_begin = p.split * keys, k_end = splits > 1 ? min(tx.len, k_begin + keys) : tx.len;
  if (splits > 1 && k_begin >= tx.len) return;  // (the join knows the text's length)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lq = lane & 31, lh = lane >> 5;
  const int rows = a.rep * a.n_q, d = a.d, r0 = p.tile * 32;
  bf16 *Ks = (bf16*)(smem + wave * AREA), *Vs = Ks + KW * LDK;
  const uint8_t* mask = a.mask ? a.mask + tx.m0 : nullptr;
  const float sl2 = a.scale == 0.f ? LOG2E : fabsf(a.scale) * LOG2E;
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;

  const int pk = lane / LPR, pc = lane % LPR * 8;
  const int ko = pc < d ? (pk * (int)a.k_ld + pc) * 2 : OOB, vo = pc < d ? (pk * (int)a.v_ld + pc) * 2 : OOB;
  const bf16* K = (const bf16*)a.k + tx.k0 + p.g * a.k_head;
  const bf16* V = (const bf16*)a.v + tx.v0 + p.g * a.v_head;
  bf16x8 rk[CPT], rv[CPT];
  auto fetch = [&](int k0, uint32_t bits) __attribute__((always_inline)) {
    const int n = min(KW, k_end - k0);
    const __amdgpu_buffer_rsrc_t kr = make_rsrc(K + (long)k0 * a.k_ld, ((n - 1) * (long)a.k_ld + d) * 2);
    const __amdgpu_buffer_rsrc_t vr = make_rsrc(V + (long)k0 * a.v_ld, ((n - 1) * (long)a.v_ld + d) * 2);
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const bool on = bits >> pk >> (RPP * i) & 1;
      rk[i] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(kr, on ? ko + i * RPP * (int)a.k_ld * 2 : OOB, 0, 0));
      rv[i] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(vr, on ? vo + i * RPP * (int)a.v_ld * 2 : OOB, 0, 0));
    }
  };
  auto own_key = [&](int k0) -> bool {
    const int k = k0 + lq;
    return k < k_end && (!mask || mask[k]);
  };
  int k0 = k_begin + wave * KW;
  uint32_t bits = (uint32_t)__ballot(own_key(k0));
  if (k0 < k_end) fetch(k0, bits);

  bf16x8 qf[NJ];
  {
    const RowAt at = row_at(a, r0 + lq);
    const bf16* Q = (const bf16*)a.q + (long)p.img * a.q_img + at.t * a.q_ld + (p.g * a.rep + at.h) * a.q_head;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = 16 * j + 8 * lh;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (r0 + lq < rows && c < d && a.scale != 0.f) v = *(const uint4*)(Q + c);
      v.x ^= flip;
      v.y ^= flip;
      v.z ^= flip;
      v.w ^= flip;
      qf[j] = __builtin_bit_cast(bf16x8, v);
    }
  }
  if constexpr (SF)  // ones in channel d of every key
    if (lane < KW) {
      bf16x8 v = {};
      v[0] = (bf16)1.0f;
      *(bf16x8*)&Vs[lane * LDV + d] = v;
    }
  bf16x8 ones = {};
  if (lh == 0) ones[0] = (bf16)1.0f;
  f32x16 o[ND];
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;

  for (; k0 < k_end; k0 += NW * KW) {
#pragma unroll
    for (int i = 0; i < CPT; ++i)
      if (pc < D16) {
        *(bf16x8*)&Ks[(pk + RPP * i) * LDK + pc] = rk[i];
        if (!SF || pc < d) *(bf16x8*)&Vs[(pk + RPP * i) * LDV + pc] = rv[i];
      }
    asm volatile("" ::: "memory");  // (one wave's LDS accesses complete in order)
    const uint32_t now = bits;
    const int kn = k0 + NW * KW;
    if (kn < k_end) {
      bits = (uint32_t)__ballot(own_key(kn));
      fetch(kn, bits);
    }
    if (!now) continue;
    const f32x16 zero = {};
    bf16x8 off = {};  // (keys that take no part start from -inf)
    if (lh == 0) off[0] = __builtin_bit_cast(bf16, (unsigned short)(now >> lq & 1 ? 0 : 0xFF80));
    f32x16 s = mfma32(off, ones, zero);
#pragma unroll
    for (int j = 0; j < NJ; ++j) s = mfma32(*(const bf16x8*)&Ks[lq * LDK + 16 * j + 8 * lh], qf[j], s);
    float v = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) v = fmaxf(v, s[r]);
    const float2 h = half_swap(v);
    const float mt = fmaxf(h.x, h.y) * sl2;
    const bool need = mt > m_run + TAU;
    if (__any(need)) {
      const float al = need ? __builtin_amdgcn_exp2f(m_run - mt) : 1.0f;
      m_run = need ? mt : m_run;
      l_run *= al;
#pragma unroll
      for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[t][r] *= al;
    }
    const float ref = exp_ref(m_run);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      // (as bf16 plus the rest as bf16, 2^-17 of each: these products have time to spare)
      bf16x8 pf, pr;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[8 * u + i], sl2, -ref));
        if constexpr (!SF) l_run += x;
        pf[i] = (bf16)x;
        pr[i] = (bf16)(x - (float)pf[i]);
      }
#pragma unroll
      for (int t = 0; t < ND; ++t) {
        const bf16* at = &Vs[(16 * u + 4 * lh + ((lane & 15) >> 2)) * LDV + t * 32 + (lane & 16) + 4 * (lane & 3)];
        const bf16x4 lo = read_transposed(at), hi = read_transposed(at + 8 * LDV);
        const bf16x8 vf = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        o[t] = mfma32(vf, pf, mfma32(vf, pr, o[t]));
      }
    }
    asm volatile("" ::: "memory");
  }

  // the wave's row sums, maxima and O to LDS
  float l = l_run;
  if constexpr (SF) {  // (d is a multiple of 8: register 0 of a quad of half 0)
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (32 * t + 8 * i == d) l = o[t][4 * i];
    l = lh == 0 ? l : 0.f;
  }
  const float2 h = half_swap(l);
  const int here = min(32, rows - r0);
  if (lh == 0) {
    sm[wave][lq] = m_run;
    sl[wave][lq] = h.x + h.y;
  }
  float* R = (float*)(smem + wave * AREA);
  if (lq < here)
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = 32 * t + 8 * i + 4 * lh;
        if (c < d) *(float4*)(R + lq * LDO + c) = make_float4(o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]);
      }
  __syncthreads();
  join_waves<bf16, NW>(a, p, splits, r0, here, (const float*)smem, AREA / 4, LDO, sm, sl);
}

// ------------------------------------------------------------------ many rows, fp32
// The same on fp32 MFMAs (32 x 32 x 2), tiles of 32 keys, a wave per 32 rows.
// Channels are summed in the order that makes a lane's share of them four
// consecutive ones (half lh takes 8 i + 4 lh + [0, 4)); a key's probability
// meets its V row straight from the register it was computed in, since the two
// k of an MFMA are the two lane halves' keys.  Bound by the fp32 matrix rate
// once the card is full; 6 x 1024 rows, 8 heads of 32 on 4, up to 231 keys (20 us,
// 37 TFLOP/s) wait for the blocks of the longest text.
namespace {
constexpr int FT = 32;
__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
#else
  return c;
#endif
}
}  // namespace

template <int D32>
__global__ __launch_bounds__(256, D32 <= 64 ? 2 : 1) void cross_f32_kernel(CrossArgs a, int keys, int tiles, int splits,
                                                                               int together) {
  constexpr int NW = 4, NI = D32 / 8, ND = D32 / 32, NT = 64 * NW, LDK = D32 + 4, LDV = D32 + 8;  // (rows apart by banks)
  constexpr int CPT = FT * (D32 / 4) / NT;
  __shared__ __attribute__((aligned(16))) float Ks[2][FT * LDK];
  __shared__ __attribute__((aligned(16))) float Vs[2][FT * LDV];
  const Place p = place_of(a.kv_heads, tiles, splits, a.n, together);
  if (!p.on) return;
  const Text tx = text_of(a, p.img);
  const int k_begin = p.split * keys, k_end = splits > 1 ? min(tx.len, k_begin + keys) : tx.len;
  if (splits > 1 && k_begin >= tx.len) return;  // (the join knows the text's length)
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lq = lane & 31, lh = lane >> 5;
  const int rows = a.rep * a.n_q, r = p.tile * (32 * NW) + wave * 32 + lq, d = a.d;
  const RowAt at = row_at(a, r);
  const int t_q = at.t, h_q = p.g * a.rep + at.h;
  const uint8_t* mask = a.mask ? a.mask + tx.m0 : nullptr;
  const float qs = a.scale * LOG2E;

  f32x4 qf[NI];
  {
    const float* Q = (const float*)a.q + (long)p.img * a.q_img + t_q * a.q_ld + h_q * a.q_head;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int c = 8 * i + 4 * lh;
      qf[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (r < rows && c < d) qf[i] = *(const f32x4*)(Q + c) * qs;
    }
  }
  f32x16 o[ND];
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  float m_run = -INFINITY, l = 0.f;

  const float* K = (const float*)a.k + tx.k0 + p.g * a.k_head;
  const float* V = (const float*)a.v + tx.v0 + p.g * a.v_head;
  uint4 rk[CPT], rv[CPT];
  auto fetch = [&](int k0, uint32_t bits) __attribute__((always_inline)) {
    const int n = min(FT, k_end - k0);
    const __amdgpu_buffer_rsrc_t kr = make_rsrc(K + (long)k0 * a.k_ld, ((n - 1) * (long)a.k_ld + d) * 4);
    const __amdgpu_buffer_rsrc_t vr = make_rsrc(V + (long)k0 * a.v_ld, ((n - 1) * (long)a.v_ld + d) * 4);
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const int idx = tid + NT * i, key = idx / (D32 / 4), c = idx % (D32 / 4) * 4;
      const bool on = (bits >> key & 1) && c < d;
      rk[i] = __builtin_bit_cast(uint4, buf_load16(kr, on ? (key * (int)a.k_ld + c) * 4 : OOB));
      rv[i] = __builtin_bit_cast(uint4, buf_load16(vr, on ? (key * (int)a.v_ld + c) * 4 : OOB));
    }
  };
  auto stage = [&](int b) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const int idx = tid + NT * i, key = idx / (D32 / 4), c = idx % (D32 / 4) * 4;
      *(uint4*)&Ks[b][key * LDK + c] = rk[i];
      *(uint4*)&Vs[b][key * LDV + c] = rv[i];
    }
  };
  auto own_key = [&](int k0) -> bool {
    const int k = k0 + lq;
    return k < k_end && (!mask || mask[k]);
  };
  if (k_begin < k_end) {
    uint32_t bits = (uint32_t)__ballot(own_key(k_begin));
    fetch(k_begin, bits);
    bool nk = own_key(k_begin + FT);
    stage(0);
    __syncthreads();
    for (int k0 = k_begin, b = 0; k0 < k_end; k0 += FT, b ^= 1) {
      uint32_t next = 0;
      const bool more = k0 + FT < k_end;
      if (more) {
        next = (uint32_t)__ballot(nk);
        fetch(k0 + FT, next);
        nk = own_key(k0 + 2 * FT);
      }
      if (bits) {
        f32x16 s = {};
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          if (8 * i >= d) break;
          const f32x4 kf = *(const f32x4*)&Ks[b][lq * LDK + 8 * i + 4 * lh];
#pragma unroll
          for (int e = 0; e < 4; ++e) s = mfma_f32(kf[e], qf[i][e], s);
        }
        // register i: key 8 (i / 4) + 4 lh + i % 4
        if (bits != ~0u) {
          const uint32_t bm = bits >> (4 * lh);
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!(bm >> (8 * (i >> 2) + (i & 3)) & 1)) s[i] = -INFINITY;
        }
        float v = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) v = fmaxf(v, s[i]);
        const float2 hv = half_swap(v);
        const float mt = fmaxf(hv.x, hv.y);
        const bool need = mt > m_run + TAU;
        if (__any(need)) {
          const float al = need ? __builtin_amdgcn_exp2f(m_run - mt) : 1.0f;
          m_run = need ? mt : m_run;
          l *= al;
#pragma unroll
          for (int t = 0; t < ND; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[t][i] *= al;
        }
        const float ref = exp_ref(m_run);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float pr = __builtin_amdgcn_exp2f(s[i] - ref);
          l += pr;
          const float* vr = &Vs[b][(8 * (i >> 2) + 4 * lh + (i & 3)) * LDV + lq];
#pragma unroll
          for (int t = 0; t < ND; ++t) o[t] = mfma_f32(vr[32 * t], pr, o[t]);
        }
      }
      if (more) stage(b ^ 1);
      __syncthreads();
      bits = next;
    }
  }
  const float2 hl = half_swap(l);
  l = hl.x + hl.y;
  if (r >= rows) return;
  float* out = (float*)a.o + (long)p.img * a.o_img + t_q * a.o_ld + h_q * a.o_head;
  float f = l == 0.f ? 0.f : 1.0f / l;
  if (splits > 1) {
    const Scratch sc = scratch_at(a, p.img, p.g, r, p.split, splits);
    if (lh == 0) {
      sc.ml[0] = m_run;
      sc.ml[1] = l;
    }
    out = sc.o;
    f = 1.0f;
  }
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = 32 * t + 8 * i + 4 * lh;
      if (c < d) *(float4*)(out + c) = make_float4(o[t][4 * i] * f, o[t][4 * i + 1] * f, o[t][4 * i + 2] * f, o[t][4 * i + 3] * f);
    }
}

// Few rows, fp32 (9 to 128; up to 8 take the lanes above): as cross_keys_kernel,
// on fp32 MFMAs.  PRE: the next keys are loaded while these are multiplied (wider
// heads have no registers left for them, and 16 times the products of a bf16 tile to hide them with).
template <int D32, int NW>
__global__ __launch_bounds__(64 * NW) void cross_keys_f32_kernel(CrossArgs a, int keys, int tiles, int splits, int together) {
  constexpr int NI = D32 / 8, ND = D32 / 32, LDK = D32 + 4, LDV = D32 + 8, LDO = D32 + 4, AREA = FT * (LDK + LDV);
  constexpr int CPT = FT * (D32 / 4) / 64;
  constexpr bool PRE = D32 <= 128;
  __shared__ __attribute__((aligned(16))) float smem[NW * AREA];
  __shared__ float sm[NW][32], sl[NW][32];
  const Place p = place_of(a.kv_heads, tiles, splits, a.n, together);
  if (!p.on) return;
  const Text tx = text_of(a, p.img);
  const int k_begin = p.split * keys, k_end = splits > 1 ? min(tx.len, k_begin + keys) : tx.len;
  if (splits > 1 && k_begin >= tx.len) return;  // (the join knows the text's length)
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lq = lane & 31, lh = lane >> 5;
  const int rows = a.rep * a.n_q, d = a.d, r0 = p.tile * 32;
  float *Ks = smem + wave * AREA, *Vs = Ks + FT * LDK;
  const uint8_t* mask = a.mask ? a.mask + tx.m0 : nullptr;
  const float qs = a.scale * LOG2E;
  const float* K = (const float*)a.k + tx.k0 + p.g * a.k_head;
  const float* V = (const float*)a.v + tx.v0 + p.g * a.v_head;

  uint4 rk[CPT], rv[CPT];
  auto load = [&](const float* X, long ld, int k0, uint32_t bits, uint4 (&r)[CPT]) __attribute__((always_inline)) {
    const int n = min(FT, k_end - k0);
    const __amdgpu_buffer_rsrc_t xr = make_rsrc(X + (long)k0 * ld, ((n - 1) * ld + d) * 4);
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const int idx = lane + 64 * i, key = idx / (D32 / 4), c = idx % (D32 / 4) * 4;
      const bool on = (bits >> key & 1) && c < d;
      r[i] = __builtin_bit_cast(uint4, buf_load16(xr, on ? (key * (int)ld + c) * 4 : OOB));
    }
  };
  auto put = [&](float* X, int ld, const uint4 (&r)[CPT]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const int idx = lane + 64 * i, key = idx / (D32 / 4), c = idx % (D32 / 4) * 4;
      *(uint4*)&X[key * ld + c] = r[i];
    }
  };
  auto own_key = [&](int k0) -> bool {
    const int k = k0 + lq;
    return k < k_end && (!mask || mask[k]);
  };
  int k0 = k_begin + wave * FT;
  uint32_t bits = (uint32_t)__ballot(own_key(k0));
  if (PRE && k0 < k_end) {
    load(K, a.k_ld, k0, bits, rk);
    load(V, a.v_ld, k0, bits, rv);
  }
  f32x4 qf[NI];
  {
    const RowAt at = row_at(a, r0 + lq);
    const float* Q = (const float*)a.q + (long)p.img * a.q_img + at.t * a.q_ld + (p.g * a.rep + at.h) * a.q_head;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int c = 8 * i + 4 * lh;
      qf[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (r0 + lq < rows && c < d) qf[i] = *(const f32x4*)(Q + c) * qs;
    }
  }
  f32x16 o[ND];
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  float m_run = -INFINITY, l = 0.f;
  for (; k0 < k_end; k0 += NW * FT) {
    if constexpr (!PRE) load(K, a.k_ld, k0, bits, rk);
    put(Ks, LDK, rk);
    if constexpr (!PRE) load(V, a.v_ld, k0, bits, rv);
    put(Vs, LDV, rv);
    asm volatile("" ::: "memory");  // (one wave's LDS accesses complete in order)
    const uint32_t now = bits;
    const int kn = k0 + NW * FT;
    if (kn < k_end) {
      bits = (uint32_t)__ballot(own_key(kn));
      if constexpr (PRE) {
        load(K, a.k_ld, kn, bits, rk);
        load(V, a.v_ld, kn, bits, rv);
      }
    }
    if (!now) continue;
    f32x16 s = {};
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      if (8 * i >= d) break;
      const f32x4 kf = *(const f32x4*)&Ks[lq * LDK + 8 * i + 4 * lh];
#pragma unroll
      for (int e = 0; e < 4; ++e) s = mfma_f32(kf[e], qf[i][e], s);
    }
    if (now != ~0u) {
      const uint32_t bm = now >> (4 * lh);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!(bm >> (8 * (i >> 2) + (i & 3)) & 1)) s[i] = -INFINITY;
    }
    float v = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) v = fmaxf(v, s[i]);
    const float2 hv = half_swap(v);
    const float mt = fmaxf(hv.x, hv.y);
    const bool need = mt > m_run + TAU;
    if (__any(need)) {
      const float al = need ? __builtin_amdgcn_exp2f(m_run - mt) : 1.0f;
      m_run = need ? mt : m_run;
      l *= al;
#pragma unroll
      for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] *= al;
    }
    const float ref = exp_ref(m_run);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float pr = __builtin_amdgcn_exp2f(s[i] - ref);
      l += pr;
      const float* vr = &Vs[(8 * (i >> 2) + 4 * lh + (i & 3)) * LDV + lq];
#pragma unroll
      for (int t = 0; t < ND; ++t) o[t] = mfma_f32(vr[32 * t], pr, o[t]);
    }
    asm volatile("" ::: "memory");
  }
  const float2 hl = half_swap(l);
  const int here = min(32, rows - r0);
  if (lh == 0) {
    sm[wave][lq] = m_run;
    sl[wave][lq] = hl.x + hl.y;
  }
  if (lq < here)
#pragma unroll
    for (int t = 0; t < ND; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = 32 * t + 8 * i + 4 * lh;
        if (c < d) *(float4*)(Ks + lq * LDO + c) = make_float4(o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]);
      }
  __syncthreads();
  join_waves<float, NW>(a, p, splits, r0, here, smem, AREA, LDO, sm, sl);
}

// ------------------------------------------------------------------ launch
template <int RB>
static void launch_few(const CrossArgs& a, const Plan& p, hipStream_t s) {
  const unsigned grid = place_blocks(a.kv_heads, 1, p.splits, a.n, 0);
  if (a.d <= 32)
    cross_few_kernel<RB, 4><<<grid, 512, 0, s>>>(a, p.keys, p.splits);
  else if (a.d <= 64)
    cross_few_kernel<RB, 8><<<grid, 512, 0, s>>>(a, p.keys, p.splits);
  else if (a.d <= 128)
    cross_few_kernel<RB, 16><<<grid, 512, 0, s>>>(a, p.keys, p.splits);
  else
    cross_few_kernel<RB, 32><<<grid, 512, 0, s>>>(a, p.keys, p.splits);
}

template <int D16, bool SF>
static void launch_bf16(const CrossArgs& a, const Plan& p, hipStream_t s) {
  const long rows = (long)a.rep * a.n_q;
  const int tiles = (int)((rows + 127) / 128);
  const int together = place_together(a, 2);
  cross_bf16_kernel<D16, SF, false><<<place_blocks(a.kv_heads, tiles, p.splits, a.n, together), 256, 0, s>>>(
      a, p.keys, tiles, p.splits, 1, together);
}

template <int D16, bool SF>
static void launch_sum(const CrossArgs& a, const Plan& p, hipStream_t s) {
  const long rows = (long)a.rep * a.n_q;
  if (p.kind <= 1) {
    constexpr int NW = 4;
    const int tiles = (int)((rows + 31) / 32);
    const int together = tiles > 1 ? place_together(a, 2) : 0;
    cross_keys_kernel<D16, SF, NW><<<place_blocks(a.kv_heads, tiles, p.splits, a.n, together), 64 * NW, 0, s>>>(a, p.keys, tiles, p.splits, together);
    return;
  }
  // (wider heads: LDS for the output rows leaves one block a CU; 16 x 1024 rows, 8
  // heads of 120, up to 120 keys 37 us against 29)
  if constexpr (D16 <= 96)
    if (a.max_len <= 2 * KT) {
      // up to 8 groups of rows per wave, as long as some 1000 blocks remain
      const long groups = (rows + 127) / 128, all = groups * a.kv_heads * a.n;
      const int passes = (int)(all / 1024 < 1 ? 1 : all / 1024 > 8 ? 8 : all / 1024);
      const int tiles = (int)((groups + passes - 1) / passes);
      cross_bf16_kernel<D16, SF, true><<<place_blocks(a.kv_heads, tiles, 1, a.n, 0), 256, 0, s>>>(a, 0, tiles, 1, passes, 0);
      return;
    }
  launch_bf16<D16, SF>(a, p, s);
}

template <int D16>
static void launch_width(const CrossArgs& a, const Plan& p, hipStream_t s) {
  if (a.d < D16)
    launch_sum<D16, true>(a, p, s);
  else
    launch_sum<D16, false>(a, p, s);
}

template <int D32>
static void launch_f32(const CrossArgs& a, const Plan& p, hipStream_t s) {
  const long rows = (long)a.rep * a.n_q;
  const int together = place_together(a, 4);
  if (p.kind == 1) {
    constexpr int NW = D32 <= 128 ? 4 : 2;  // (as many as the LDS holds)
    const int tiles = (int)((rows + 31) / 32);
    const unsigned grid = place_blocks(a.kv_heads, tiles, p.splits, a.n, together);
    if (a.max_len <= FT)  // (the first wave has them all: the same sums; 13 x 22 rows, 40 heads of 128 on 10: 28 -> 19 us)
      cross_keys_f32_kernel<D32, 1><<<grid, 64, 0, s>>>(a, p.keys, tiles, p.splits, together);
    else
      cross_keys_f32_kernel<D32, NW><<<grid, 64 * NW, 0, s>>>(a, p.keys, tiles, p.splits, together);
  } else {
    const int tiles = (int)((rows + 127) / 128);
    cross_f32_kernel<D32><<<place_blocks(a.kv_heads, tiles, p.splits, a.n, together), 256, 0, s>>>(a, p.keys, tiles, p.splits, together);
  }
}

long cross_attention_scratch_floats(DType dt, int n, int heads, int kv_heads, int d, int n_q, int max_len) {
  const Plan p = plan_of(heads / kv_heads, n_q, max_len);
  // (a grid holds less than 2^32 threads: blocks of at most 512 per 32 rows of a
  // K/V head and split, in eights, and joins of 64 a row)
  const double rows = (double)heads * n_q * n, tiles = (double)heads / kv_heads * n_q / 32 + 1;
  const double blocks = ((double)n * kv_heads + 8) * tiles * p.splits, shared = (tiles * p.splits * n + 8) * kv_heads;
  if (blocks * 512 > 4.0e9 || shared * 512 > 4.0e9 || (p.splits > 1 && rows * 64 > 4.0e9)) return -1;
  return p.splits > 1 ? (long)rows * p.splits * (d + 2) : 0;
}

hipError_t launch_cross_attention(DType dt, CrossArgs a, hipStream_t s) {
  const long rows = (long)a.rep * a.n_q;
  if (a.n <= 0 || rows <= 0) return hipSuccess;
  const Plan p = plan_of(a.rep, a.n_q, a.max_len);
  if (p.splits > 1 && !a.scratch) return hipErrorInvalidValue;
  if (a.rep > 1) {  // r = q rep + s, r < 2^31: with l = ceil(log2 rep), mul = ceil(2^(31 + l) / rep), q = r mul >> (31 + l)
    int l = 0;
    while ((1u << l) < (unsigned)a.rep) ++l;
    a.rep_mul = (unsigned)(((1ull << (31 + l)) + a.rep - 1) / a.rep);
    a.rep_shift = l - 1;
  }
  if (p.kind == 0 && dt != BF16) {
    const long r = rows;
    r == 1 ? launch_few<1>(a, p, s) : r == 2 ? launch_few<2>(a, p, s) : r <= 4 ? launch_few<4>(a, p, s) : launch_few<8>(a, p, s);
  } else if (dt == BF16) {
    if (a.d <= 32) launch_width<32>(a, p, s);
    else if (a.d <= 48) launch_width<48>(a, p, s);
    else if (a.d <= 64) launch_width<64>(a, p, s);
    else if (a.d <= 80) launch_width<80>(a, p, s);
    else if (a.d <= 96) launch_width<96>(a, p, s);
    else if (a.d <= 128) launch_width<128>(a, p, s);
    else if (a.d <= 160) launch_width<160>(a, p, s);
    else if (a.d <= 192) launch_width<192>(a, p, s);
    else launch_width<256>(a, p, s);
  } else {
    if (a.d <= 32) launch_f32<32>(a, p, s);
    else if (a.d <= 64) launch_f32<64>(a, p, s);
    else if (a.d <= 96) launch_f32<96>(a, p, s);
    else if (a.d <= 128) launch_f32<128>(a, p, s);
    else if (a.d <= 160) launch_f32<160>(a, p, s);
    else if (a.d <= 192) launch_f32<192>(a, p, s);
    else launch_f32<256>(a, p, s);
  }
  if (p.splits > 1) {
    if (dt == BF16)
      launch_join<bf16>(a, p, s);
    else
      launch_join<float>(a, p, s);
  }
  return hipGetLastError();
}

}  // namespace sd
