// Attention inside texts of their own lengths:
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(f(scale q_i . k_j) + bias(j - i))
// over the keys j of query i's own text that take part: f is the identity or
// cap tanh(. / cap), bias a table per head by distance, constant past its ends,
// less a slope times the distance; a causal text shows query i the keys up to i,
// and those of its prefix.
//
// A block takes 128 queries of one head and passes over their text's keys once,
// a wave per 32 queries.  Scores are held transposed, S^T = K Q^T, so that a
// lane has one query: its order, maximum and rescale are per lane, and P^T feeds
// O^T = V^T P^T from the registers.  What depends on the distance alone is the
// same along a diagonal: a tile's 64 x 128 values are 191, kept in LDS.
// Tiles wholly behind the causal border are passed over, and keys that a mask or
// the text's end leaves out are never read.
#include "attention_tile.h"
#include "device_common.h"
#include "kernels.h"

namespace sd {

namespace {

constexpr int TQ = 128;  // queries per block, 32 a wave

// Text c: its first row (elements of q, k, v, o; mask byte), its length, and the
// keys that all its queries see.
struct Span {
  long q0, k0, v0, o0, m0;
  int len, prefix;
};
__device__ __forceinline__ Span span_of(const TextArgs& a, int c) {
  Span t;
  if (a.start) {
    const long lo = min(max((long)a.start[c], 0L), a.tokens), hi = min(max((long)a.start[c + 1], lo), a.tokens);
    t.q0 = lo * a.q_ld;
    t.k0 = lo * a.k_ld;
    t.v0 = lo * a.v_ld;
    t.o0 = lo * a.o_ld;
    t.m0 = lo;
    t.len = (int)min(hi - lo, (long)a.max_len);
  } else {
    t.q0 = (long)c * a.q_img;
    t.k0 = (long)c * a.k_img;
    t.v0 = (long)c * a.v_img;
    t.o0 = (long)c * a.o_img;
    t.m0 = (long)c * a.max_len;
    t.len = a.length ? min(max(a.length[c], 0), a.max_len) : a.max_len;
  }
  t.prefix = a.prefix ? min(max(a.prefix[c], 0), t.len) : 0;
  return t;
}

// Block -> (text, head, tile).  Consecutive blocks go to the 8 XCDs in turn, each
// with an L2 of its own.  `chunk` tiles of all heads that share a K/V head stay
// on one XCD, next to each other in time, since they read the same keys; the
// chunks furthest into their texts come first, as a causal one costs as much as
// the keys before it.  The grid is (8 XCDs x tiles and heads of a chunk, text and K/V
// head in eights, chunk): a division costs some 40 instructions before the first load.
struct Place {
  int c, g, h, tile;
  bool on;
};
__device__ __forceinline__ Place place_of(const TextArgs& a) {
  const unsigned in = blockIdx.x >> 3, w = blockIdx.y * 8 + (blockIdx.x & 7);
  Place p;
  p.on = w < (unsigned)a.n * a.kv_heads;
  p.c = w / (unsigned)a.kv_heads;
  p.g = w - p.c * a.kv_heads;
  const unsigned t = a.rep == 1 ? in : in / (unsigned)a.rep;
  p.h = p.g * a.rep + in - t * a.rep;
  p.tile = (int)((a.chunks - blockIdx.z) * a.chunk - 1 - t);
  return p;
}

// The rows of packed texts' o that lie in no text, zeroed by the blocks of the
// first and the last one, and those of a text that is longer than max_len says
// (16 bytes a thread).
template <typename T>
__device__ __forceinline__ void zero_rest(const TextArgs& a, const Place& p) {
  constexpr int E = 16 / sizeof(T);
  const int per = a.d / E;
  auto span = [&](long lo, long hi) {
    T* o = (T*)a.o + p.h * a.o_head;
    for (long r0 = lo + (long)p.tile * TQ; r0 < hi; r0 += (long)a.chunks * a.chunk * TQ)
      for (int x = threadIdx.x; x < TQ * per; x += blockDim.x) {
        const long r = r0 + x / per;
        if (r < hi) *(uint4*)(o + r * a.o_ld + x % per * E) = make_uint4(0, 0, 0, 0);
      }
  };
  const long lo = min(max((long)a.start[p.c], 0L), a.tokens);
  span(lo + a.max_len, min((long)a.start[p.c + 1], a.tokens));
  if (p.c == 0) span(0, min((long)max(a.start[0], 0), a.tokens));
  if (p.c == a.n - 1) span(max((long)a.start[a.n], 0L), a.tokens);
}

// bias(j - i) at distance `far` in log2 units, over `unit`, from what the table holds
// there.  Finite values stay finite: up to 2^126 of either unit, past any score, and
// sums of two do not pass fp32.
__device__ __forceinline__ float table_at(const TextArgs& a, int h, int far) {
  return a.bias ? a.bias[(long)h * (2 * a.reach + 1) + min(max(far, -a.reach), a.reach) + a.reach] : 0.f;
}
__device__ __forceinline__ float term_of(float v, int far, float slope, float unit) {
  v = fmaf(-slope, fabsf((float)far), v);
  const float lim = 0x1p125f * fminf(unit, 1.f);
  if (v < -lim && v != -INFINITY) v = -lim;
  if (v > lim && v != INFINITY) v = lim;
  return v * LOG2E / unit;
}

__device__ __forceinline__ bool lanes(uint64_t bits) {  // this lane's bit
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_inverse_ballot_w64(bits);
#else
  return false;
#endif
}

// The larger one, NaN if either is.
__device__ __forceinline__ float larger(float a, float b) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_elementwise_maximum(a, b);
#else
  return a;
#endif
}

}  // namespace

// ------------------------------------------------------------------ bf16
// Slots of a key's CH 16-byte chunks in LDS, where the loads put them next to each
// other without gaps: chunk c of key r lies in slot c ^ k_swz(r) (K, whose fragment
// reads take 16 keys at one chunk) or c ^ v_swz(r) (V, whose transposing reads take
// 4 keys at four chunks), so that either set is spread over all 16 columns of 16
// bytes.  (32 chunks: over 8, so that rows 8 apart are turned alike.)
__host__ __device__ constexpr int k_low(int ch) { return (ch == 32 ? 8 : ch % 16 == 0 ? 16 : ch % 8 == 0 ? 8 : ch % 4 == 0 ? 4 : 2) - 1; }
__host__ __device__ constexpr int v_low(int ch) { return (ch % 16 == 0 ? 16 : ch % 8 == 0 ? 8 : 1) - 1; }
template <int CH>
__device__ __forceinline__ int k_swz(int r) {
  constexpr int L = k_low(CH);
  return (CH == 32 || L == 15 ? r : L == 7 ? r >> 1 : L == 3 ? r >> 2 : r >> 3) & L;
}
template <int CH>
__device__ __forceinline__ int v_swz(int r) {
  constexpr int L = v_low(CH);
  return L == 15 ? 4 * (r & 3) : L == 7 ? 2 * (r & 2) : 0;
}

// D16: head width rounded up to a width the kernel is built for.  BIAS: there is
// a term by distance.  CAP: scores are capped.  Tiles of 64 keys go from memory
// straight to LDS, one tile ahead of the one in work; a tile's K fragments, and the first
// half of V's, are read ahead of the products that use them.
// SHORT: no text is longer than the two tiles that LDS holds.  They are loaded at
// once and nothing waits afterwards; a block is as long as its chain of latencies,
// so four blocks share a CU where registers allow, which leaves fewer for fragments
// read ahead, and three for capped scores without a term, whose exponents all live at
// once.  The sums are the same.  (us, kernels of 20 heads, this form and the other; causal
// prompts of 5 to 77 tokens, 48 of them: 32 channels 7.9 and 8.8, 64 9.1 and 11.8, 128 16.9
// and 18.0, 256 48 and 57; capped 9.3 and 11.4, 12.2 and 13.1 (four blocks: 16.0), 18.6 and
// 19.7, 68 and 84; 64 texts of 128 tokens 15.0 and 16.3, 18.1 and 19.4, 33.9 and 33.6, 102 and
// 143; capped 18.4 and 19.1, 21.8 and 22.0 (four blocks: 33.2), 35.4 and 35.6, 143 and 199;
// 192 channels 72.5 and 69.4, else as 128.)
// What bounds it: a wave's vector instructions (some 9 a score without a cap, 12 with,
// the exponentials two turns each) and its products one after the other, which only
// other waves overlap.  30 calls after each other on inputs that change: 6 documents of
// 500 to 8192 tokens, 16 heads of 128 on 4, capped 1331 us, 476 TFLOP/s, vector ALU busy
// 61 %, matrix unit 34 % (the clock falls under it: 1046 us between other work); 12 texts
// of 700 to 2500, 10 heads of 80 175 us, 359 TFLOP/s, 45 %, 26 % and a third of the time
// waiting for the next tile.  (Waiting for every fragment where it is used cost a quarter more.)
// Registers: one wave per SIMD past 128 channels.  At 256 every form spills 15 to 101 of
// them, and is far off for it: 8 heads on 4 over the documents above, capped 3696 us, 171
// TFLOP/s.  At 64 the SHORT forms with a term spill 2.  No other form does.
template <int D16, bool BIAS, bool CAP, bool SHORT>
__global__ __launch_bounds__(256, D16 <= 64 ? (SHORT && (BIAS || !CAP) ? 4 : 3) : D16 <= 128 ? 2 : 1) void text_bf16_kernel(TextArgs a) {
  constexpr int NW = 4, KT = 64, NJ = D16 / 16, ND = (D16 + 31) / 32, CH = D16 / 8, NI = (CH + NW - 1) / NW, LDR = D16 + 8;
  constexpr int TILE = KT * D16;
  static_assert(NW * 32 * LDR <= 4 * TILE, "the result's rows take the place of the tiles");
  // K, K, V, V (the last rows of V are read past their end where D16 % 32)
  __shared__ __attribute__((aligned(1024))) bf16 smem[4 * TILE + 64];
  __shared__ float strip[BIAS ? 2 : 1][BIAS ? KT + TQ : 1];
  __shared__ int odd[3];  // tile i: an infinity or NaN in V where the border passes (slot i % 3)
  const Place p = place_of(a);
  if (!p.on) return;
  if (a.zero && a.start) zero_rest<bf16>(a, p);
  const Span tx = span_of(a, p.c);
  const int b0 = p.tile * TQ, d = a.d;
  const int rows = a.zero && !a.start ? a.max_len : tx.len;  // (padded rows past the text get zeros)
  if (b0 >= rows) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lq = lane & 31, lh = lane >> 5;
  const int r0 = b0 + wave * 32;
  int k_end = b0 < tx.len ? tx.len : 0;
  if (a.causal) k_end = min(k_end, max(b0 + TQ, tx.prefix));
  const int lim = a.causal ? max(r0 + lq + 1, tx.prefix) : tx.len;               // keys that this lane's query sees
  const int lim_lo = a.causal ? max(r0 + 1, tx.prefix) : tx.len;                 // ... that all of the wave's see
  const int lim_hi = r0 >= tx.len ? 0 : a.causal ? max(r0 + 32, tx.prefix) : tx.len;  // ... that any does
  const int border = a.causal ? max(b0 + 1, tx.prefix) : 0x7FFFFFFF;             // ... that all of the block's see
  const uint8_t* mask = a.mask ? a.mask + tx.m0 : nullptr;
  // (a scale of 0 or below: uniform scores, or -q, under a positive one)
  const float mag = a.scale == 0.f ? 1.f : fabsf(a.scale), sl2 = mag * LOG2E;
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
  // cap tanh(x / cap) = cap - 2 cap / (1 + exp(2 x / cap)), in log2 units
  const float c_in = CAP ? 2.f * sl2 / a.cap : 0.f, c_out = CAP ? a.cap * LOG2E : 0.f;
  auto capped = [&](float x, float add) __attribute__((always_inline)) {  // (add: c_out and what else is added)
    return fmaf(-2.f * c_out, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * c_in)), add);
  };
  // Q^T fragments (B operand): query r0 + lq, channels 16 j + 8 lh + [0, 8), as loaded
  // (their sign comes behind the first tile's loads, or those would wait for them)
  uint4 qv[NJ];
  {
    const bf16* Q = (const bf16*)a.q + tx.q0 + (long)r0 * a.q_ld + p.h * a.q_head;
    const int n = a.scale == 0.f ? 0 : min(32, tx.len - r0);
    const __amdgpu_buffer_rsrc_t qr = make_rsrc(Q, n <= 0 ? 0 : ((n - 1) * (long)a.q_ld + d) * 2);
#pragma unroll
    for (int j = 0; j < NJ; ++j)
      qv[j] = __builtin_bit_cast(uint4, buf_load16(qr, 16 * j + 8 * lh < d ? (lq * (int)a.q_ld + 16 * j + 8 * lh) * 2 : OOB));
  }
  f32x16 o[ND];
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  if (tid < 3) odd[tid] = 0;
  wait_lgkm0();
  stage_barrier();

  // Load i of this wave moves chunks 64 (wave + NW i) + lane of a tile: key, and
  // byte offsets in K and V.  (Offsets past a resource's end, as those of channels
  // from d on and of keys that take no part, write zeros.)
  const bf16* K = (const bf16*)a.k + tx.k0 + p.g * a.k_head;
  const bf16* V = (const bf16*)a.v + tx.v0 + p.g * a.v_head;
  // Where CH is a power of two, load i has load 0's slots, 256 / CH keys on.
  constexpr bool EVEN = 256 % CH == 0;
  constexpr int NO = EVEN ? 1 : NI, STEP = 256 / CH;
  int lkey[NO], ko[NO], vo[NO];
#pragma unroll
  for (int i = 0; i < NO; ++i) {
    const int q = 64 * (wave + NW * i) + lane, r = q / CH, slot = q - r * CH, kc = (slot ^ k_swz<CH>(r)) * 8, vc = (slot ^ v_swz<CH>(r)) * 8;
    lkey[i] = r & 63;  // (past the tile where NW does not divide CH: not issued)
    ko[i] = kc < d ? (r * (int)a.k_ld + kc) * 2 : OOB;
    vo[i] = vc < d ? (r * (int)a.v_ld + vc) * 2 : OOB;
  }
  auto load = [&](const bf16* base, long ld, const int (&off)[NO], bf16* to, int k0, uint64_t bits) __attribute__((always_inline)) {
    const int n = min(KT, k_end - k0);
    const rsrc4 res = resource(base + (long)k0 * ld, ((n - 1) * ld + d) * 2);
    const bool all = !~bits;
    const uint64_t mine = EVEN ? bits >> lkey[0] : 0;
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (CH % NW == 0 || wave + NW * i < CH) {
        int at = EVEN ? off[0] + i * STEP * (int)ld * 2 : off[EVEN ? 0 : i];
        if (EVEN && off[0] < 0) at = OOB;
        if (!all && !((EVEN ? mine >> (STEP * i & 63) : bits >> lkey[EVEN ? 0 : i]) & 1)) at = OOB;
        to_lds16(res, to + 512 * (wave + NW * i), at);
      }
  };
  // A key's V reaches every query of a tile, with a weight of 0 behind the causal
  // border: 0 times an infinity or NaN is NaN.  So those are taken out of a tile that the border
  // passes (by the wave whose loads brought them, once they have landed), and
  // added where they are seen.
  auto clean = [&](bf16* Vt, int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (CH % NW == 0 || wave + NW * i < CH) {
        bf16* at = Vt + 512 * (wave + NW * i) + 8 * lane;
        bf16x8 v = *(const bf16x8*)at;
        if (odd8(__builtin_bit_cast(uint4, v))) {
          odd[slot] = 1;
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (odd_f((float)v[e])) v[e] = (bf16)0.f;
          *(bf16x8*)at = v;
        }
      }
  };
  // strip[e] of the tile at k0: the term at distance k0 - b0 + e - (TQ - 1), loaded and then made
  const float slope = BIAS && a.slope ? a.slope[p.h] : 0.f;
  auto far_of = [&](int k0) { return k0 - b0 + min(tid, KT + TQ - 2) - (TQ - 1); };
  auto strip_set = [&](int b, int k0, float v) __attribute__((always_inline)) {
    if (tid < KT + TQ - 1) strip[BIAS ? b : 0][BIAS ? tid : 0] = term_of(v, far_of(k0), slope, CAP ? 1.f : sl2);
  };
  // which of the 64 keys from k0 on take part: lane's own mask byte, as loaded; then a bit per key
  const __amdgpu_buffer_rsrc_t mr = make_rsrc(mask, k_end);
  auto own_mask = [&](int k0) -> int {
    return mask ? (int)__builtin_amdgcn_raw_buffer_load_b8(mr, k0 + lane, 0, 0) : 1;
  };
  auto ballot = [&](int k0, int own) -> uint64_t { return __ballot(k0 + lane < k_end && own); };

  // K fragment of slice j: chunk 2 j + lh of key lq, V fragment t: keys 4 lh + (lane % 16) / 4
  // and 8 on, channels 32 t + (lane & 16) on.  A slot is the chunk's number with
  // some of its low bits turned, so both addresses are one xor and a constant away.
  constexpr int KL = k_low(CH), VL = v_low(CH);
  const int k_at = lq * D16 + (lh ^ k_swz<CH>(lq)) * 8;
  const int vr0 = 4 * lh + ((lane & 15) >> 2);
  const int v_at = vr0 * D16 + ((((lane & 16) >> 3) + ((lane & 3) >> 1)) ^ v_swz<CH>(vr0)) * 8 + 4 * (lane & 1);
  auto k_frag = [&](const bf16* Kb, int kt, int j) __attribute__((always_inline)) {
    return *(const bf16x8*)(Kb + (k_at ^ ((2 * j & KL) * 8)) + (2 * j & ~KL) * 8 + kt * 32 * D16);
  };
  auto v_frag = [&](const bf16* Vb, int u, int t) __attribute__((always_inline)) {
    const bf16* at = Vb + (v_at ^ ((4 * t & VL) * 8)) + (4 * t & ~VL) * 8 + 16 * u * D16;
    const bf16x4 lo = read_transposed(at), hi = read_transposed(at + 8 * D16);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // A masked key's score becomes -inf by a select, or (ADD) by a product that adds it,
  // and by the select only in a wave that the sum leaves with a NaN: 0 times an infinite q
  // and a term of +inf or NaN are in it.  (us, added and selected: 16 texts of 200 to 512,
  // 20 heads of 64, no masks 30.1 and 29.4, masks 31.7 and 34.5, masks and bias 36.6 and 39.2;
  // two causal texts of 3000 and 4000, 16 heads of 128 148 and 140, of 192 355 and 327, masks
  // at 128 37.5 and 39.9; 8 heads of 256, 1500 and 2000 tokens 235 and 288; 48 prompts with
  // masks, 20 heads of 64 12.0 and 10.2.)
  constexpr bool ADD = !CAP && (D16 > 192 || (!SHORT && D16 <= 96));
  bf16x8 ones = {};  // B operand of that product: ones for k = 0
  if (ADD && lh == 0) ones[0] = (bf16)1.0f;
  const int sb = TQ - 1 - wave * 32 - lq + 4 * lh;  // strip's element at key 4 lh for this lane's query

  // Register r of half kt of a tile's scores: key 32 kt + 8 (r / 4) + 4 lh + r % 4.
  // What they start from: the term by distance, and (ADD) -inf for masked keys
  // (one product of a column of 0 or -inf per key with a row of ones).
  auto start = [&](f32x16 (&s)[2], int b, uint64_t bits) __attribute__((always_inline)) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kt][r] = BIAS && !CAP ? strip[b][sb + 32 * kt + 8 * (r >> 2) + (r & 3)] : 0.f;
    if (ADD && mask && ~bits)
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        bf16x8 off = {};
        if (lh == 0) off[0] = __builtin_bit_cast(bf16, (unsigned short)(bits >> (32 * kt + lq) & 1 ? 0 : 0xFF80));
        s[kt] = mfma32(off, ones, s[kt]);
      }
  };
  // -inf for keys that the mask leaves out, whatever their scores became: a select each,
  // whose lanes are made of two bits on the scalar unit.
  auto leave_out = [&](f32x16 (&s)[2], uint64_t bits) __attribute__((always_inline)) {
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const uint32_t w = (uint32_t)(bits >> (32 * kt));
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int c = 8 * (r >> 2) + (r & 3);
        const uint32_t lo = (uint32_t)((int)(w << (31 - c)) >> 31), hi = (uint32_t)((int)(w << (27 - c)) >> 31);
        s[kt][r] = lanes(lo | (uint64_t)hi << 32) ? s[kt][r] : -INFINITY;
      }
    }
  };
  // What was taken out of V, added for the queries that see it (a weight above 0 times it is itself).
  auto add_odd = [&](uint64_t bits, int k0) __attribute__((always_inline)) {
#pragma unroll 1
    for (int j = 0; j < KT; ++j) {
      if (!(bits >> j & 1)) continue;
      const __amdgpu_buffer_rsrc_t vr = make_rsrc(V + (long)(k0 + j) * a.v_ld, d * 2);
      const bool seen = k0 + j < lim;
#pragma unroll
      for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint2 w = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(vr, (32 * t + 8 * i + 4 * lh) * 2, 0, 0));
          const bf16x4 x = __builtin_bit_cast(bf16x4, w);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[t][4 * i + e] += seen && odd_f((float)x[e]) ? (float)x[e] : 0.f;
        }
    }
  };

  if (k_end > 0) {
    int own = own_mask(0), own1 = own_mask(KT);
    float f = BIAS ? table_at(a, p.h, far_of(0)) : 0.f, f1 = BIAS && SHORT ? table_at(a, p.h, far_of(KT)) : 0.f;
    uint64_t bits = ballot(0, own), next = 0;
    load(K, a.k_ld, ko, smem, 0, bits);
    load(V, a.v_ld, vo, smem + 2 * TILE, 0, bits);
    if (SHORT && KT < k_end) {
      next = ballot(KT, own1);
      load(K, a.k_ld, ko, smem + TILE, KT, next);
      load(V, a.v_ld, vo, smem + 3 * TILE, KT, next);
    }
    if constexpr (BIAS) strip_set(0, 0, f);
    if constexpr (BIAS && SHORT) strip_set(1, KT, f1);
    wait_vmcnt<0>();
    if (KT > border) clean(smem + 2 * TILE, 0);
    if (SHORT && KT < k_end && 2 * KT > border) clean(smem + 3 * TILE, 1);
    wait_lgkm0();
    stage_barrier();
    bf16x8 qf[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      qv[j].x ^= flip;
      qv[j].y ^= flip;
      qv[j].z ^= flip;
      qv[j].w ^= flip;
      qf[j] = __builtin_bit_cast(bf16x8, qv[j]);
    }
    own = own1;
    for (int k0 = 0, t = 0, slot = 0; k0 < k_end; k0 += KT, t ^= 1) {
      const int s1 = slot == 2 ? 0 : slot + 1;
      if constexpr (!SHORT) {
        next = ballot(k0 + KT, own);
        if (k0 + KT < k_end) {  // (what the registers get is waited for at the end of the tile, with the rest)
          if (BIAS) f = table_at(a, p.h, far_of(k0 + KT));
          own = own_mask(k0 + 2 * KT);
          load(K, a.k_ld, ko, smem + (t ^ 1) * TILE, k0 + KT, next);
          load(V, a.v_ld, vo, smem + (2 + (t ^ 1)) * TILE, k0 + KT, next);
        }
      }
      const bf16 *Kb = smem + t * TILE, *Vb = smem + (2 + t) * TILE;
      if (k0 < lim_hi) {  // (uniform in a wave)
        // Fragments are read ahead of the products that use them, K's all at once,
        // V's two slices at a time, the first ones before the softmax.
        f32x16 s[2];
        {
          bf16x8 kf[2][NJ];
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int j = 0; j < NJ; ++j) kf[kt][j] = k_frag(Kb, kt, j);
          start(s, t, bits);
          if constexpr (!SHORT) __builtin_amdgcn_sched_barrier(0);
          __builtin_amdgcn_s_setprio(1);  // (before the other waves' softmax: 1133 -> 1118 us on long capped documents)
#pragma unroll
          for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) s[kt] = mfma32(kf[kt][j], qf[j], s[kt]);
          __builtin_amdgcn_s_setprio(0);
        }
        bf16x8 vf[2][ND];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < ND; ++i) vf[u][i] = v_frag(Vb, u, i);
        if constexpr (!SHORT) __builtin_amdgcn_sched_barrier(0);
        const bool part = k0 + KT > lim_lo, gaps = mask && ~bits;
        const bool late = CAP && !BIAS && !part && !gaps;  // whole tiles without a term: the cap is taken with the exponents
        if (CAP && !late)
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              s[kt][r] = capped(s[kt][r], BIAS ? c_out + strip[t][sb + 32 * kt + 8 * (r >> 2) + (r & 3)] : c_out);
        // the causal border and the text's end
        if (part) {
          const int left = lim - k0 - 4 * lh;
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int c = 32 * kt + 8 * (r >> 2) + (r & 3);
              if (c >= left) s[kt][r] = -INFINITY;
            }
        }
        if (!ADD && gaps) leave_out(s, bits);
        auto largest = [&] {
          float v = s[0][0];
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) v = ADD ? larger(v, s[kt][r]) : fmaxf(v, s[kt][r]);
          return v;
        };
        float v = largest();
        if (ADD && gaps && __any(v != v)) {
          leave_out(s, bits);
          v = largest();
        }
        const float2 h = half_swap(v);
        float mt = fmaxf(h.x, h.y);
        if constexpr (!CAP) mt *= sl2;
        else if (late) mt = capped(mt, c_out);  // (the cap keeps the order of scores)
        const bool need = mt > m_run + TAU;
        if (__any(need)) {  // (where a row's maximum stays, its sums are multiplied by one)
          const float al = need ? __builtin_amdgcn_exp2f(m_run - mt) : 1.0f;
          m_run = need ? mt : m_run;
          l_run *= al;
#pragma unroll
          for (int t2 = 0; t2 < ND; ++t2)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[t2][r] *= al;
        }
        const float ref = exp_ref(m_run);
        // (the exponent is s sl2 - ref in one rounding; past 2^20 the one that ref
        // holds of its own product would no longer be a small part of a step.  Each query by
        // itself: another's ref may come from a key that this one does not see)
        float mul = sl2;
        const bool far = fabsf(ref) > 0x1p20f;
        if (!CAP && __any(far)) {
          const float by = far ? sl2 : 1.f;
          mul = far ? 1.f : sl2;
#pragma unroll
          for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kt][r] *= by;
        }
        if constexpr (CAP) {
          if (late) {
            const float add = c_out - ref;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
              for (int r = 0; r < 16; ++r) s[kt][r] = capped(s[kt][r], add);
          } else {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
              for (int r = 0; r < 16; ++r) s[kt][r] -= ref;
          }
        }
        auto probs = [&](int u) __attribute__((always_inline)) {
          bf16x8 pf;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float x = s[u >> 1][8 * (u & 1) + i];
            pf[i] = (bf16)__builtin_amdgcn_exp2f(CAP ? x : fmaf(x, mul, -ref));
          }
          l_run = sum_probs(pf, l_run);
          return pf;
        };
        // O^T += V^T P^T, 16 keys at a time: slot (lh, i) of slice u is key 16 u +
        // 8 (i / 4) + 4 lh + i % 4, register 8 (u % 2) + i of half u / 2.  The
        // probabilities are rounded to bf16 (by up to 2^-8 of each, half a step) and
        // summed as rounded, so that the rounding cancels where one key prevails.
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const bf16x8 pf = probs(u);
#pragma unroll
          for (int i = 0; i < ND; ++i) o[i] = mfma32(vf[u & 1][i], pf, o[i]);
          if (u < 2) {
#pragma unroll
            for (int i = 0; i < ND; ++i) vf[u][i] = v_frag(Vb, u + 2, i);
            if constexpr (!SHORT) __builtin_amdgcn_sched_barrier(0);
          }
        }
        if (k0 + KT > border && odd[slot]) add_odd(bits, k0);
      }
      bits = next;
      slot = s1;
      if constexpr (!SHORT) {
        if constexpr (BIAS) strip_set(t ^ 1, k0 + KT, f);
        wait_vmcnt<0>();
        if (k0 + 2 * KT > border && k0 + KT < k_end) clean(smem + (2 + (t ^ 1)) * TILE, s1);
        if (tid == 0) odd[s1 == 2 ? 0 : s1 + 1] = 0;  // (read before the last barrier, set after the next)
        wait_lgkm0();
        stage_barrier();
      }
    }
    if constexpr (SHORT) stage_barrier();  // (the result's rows take the place of the tiles)
  }

  // O^T: lane holds channels 32 t + 8 (r / 4) + 4 lh + r % 4 of its query.  Rows are
  // laid out in LDS (the tiles are done with) and leave 16 bytes a lane.
  const float2 h = half_swap(l_run);
  const float l = h.x + h.y, inv = l == 0.f ? 0.f : 1.0f / l;
  const bool live = r0 + lq < tx.len;
  bf16* R = smem + wave * 32 * LDR;
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = 32 * t + 8 * i + 4 * lh;
      if (c < d) {
        bf16x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (bf16)(live ? o[t][4 * i + e] * inv : 0.f);
        *(bf16x4*)(R + lq * LDR + c) = w;
      }
    }
  asm volatile("" ::: "memory");  // (one wave's LDS accesses complete in order)
  constexpr int LPR = D16 <= 32 ? 4 : D16 <= 64 ? 8 : D16 <= 128 ? 16 : 32;  // lanes a row
  const int c = lane % LPR * 8, row0 = lane / LPR;
  if (c < d) {
    bf16* O = (bf16*)a.o + tx.o0 + (long)r0 * a.o_ld + p.h * a.o_head + c;
#pragma unroll
    for (int i = 0; i < 32; i += 64 / LPR)
      if (r0 + row0 + i < rows) *(bf16x8*)(O + (row0 + i) * (int)a.o_ld) = *(const bf16x8*)(R + (row0 + i) * LDR + c);
  }
}

// ------------------------------------------------------------------ fp32
// tanh to 3e-7 of it: from |x| = 0.6 on 1 - 2 / (1 + e^2|x|), below that x + x^3 (c1 +
// c2 x^2 + ..) of least largest relative error (points of a Chebyshev grid, reweighted
// by their errors until those are level).  A third of the library function's
// instructions, which took half of a capped tile's time.
__device__ __forceinline__ float tanh_f32(float x) {
  constexpr float C1 = -0.33333298563957214f, C2 = 0.13331924378871918f, C3 = -0.053783830255270004f,
                  C4 = 0.020795971155166626f, C5 = -0.005895158275961876f;
  const float y = x * x, m = fabsf(x);
  const float lo = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, C5, C4), C3), C2), C1), x);
  const float e = __builtin_amdgcn_exp2f(m * (2.f * LOG2E));
  const float hi = copysignf(fmaf(-2.f, __builtin_amdgcn_rcpf(1.f + e), 1.f), x);
  return m < 0.6f ? lo : hi;  // (NaN takes the second)
}

// The same on fp32 MFMAs (32 x 32 x 2), tiles of 32 keys.  Channels are summed in
// the order that makes a lane's share of them four consecutive ones (half lh
// takes 8 i + 4 lh + [0, 4)); a key's probability meets its V row straight from the
// register it was computed in, since the two k of an MFMA are the two lane halves' keys.
// Few texts wait for the tiles of the longest one, a wave's 32 products of 64 cycles
// a tile at 32 channels: 6 texts of 8 to 231 tokens, 8 heads of 32, capped 25.8 us; one
// text of 4000, 8 heads of 64, causal 354 us.  One wave per SIMD past 64 channels.
template <int D32>
__global__ __launch_bounds__(256, D32 <= 64 ? 2 : 1) void text_f32_kernel(TextArgs a) {
  constexpr int NW = 4, KT = 32, NI = D32 / 8, ND = D32 / 32, NT = 64 * NW, LDK = D32 + 4, LDV = D32 + 8;  // (rows apart by banks)
  constexpr int CPT = KT * (D32 / 4) / NT;
  __shared__ __attribute__((aligned(16))) float Ks[2][KT * LDK];
  __shared__ __attribute__((aligned(16))) float Vs[2][KT * LDV];
  __shared__ float strip[2][KT + TQ];
  __shared__ int odd[3];
  const Place p = place_of(a);
  if (!p.on) return;
  if (a.zero && a.start) zero_rest<float>(a, p);
  const Span tx = span_of(a, p.c);
  const int b0 = p.tile * TQ, d = a.d;
  const int rows = a.zero && !a.start ? a.max_len : tx.len;
  if (b0 >= rows) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lq = lane & 31, lh = lane >> 5;
  const int r0 = b0 + wave * 32, r = r0 + lq;
  int k_end = b0 < tx.len ? tx.len : 0;
  if (a.causal) k_end = min(k_end, max(b0 + TQ, tx.prefix));
  const int lim = a.causal ? max(r + 1, tx.prefix) : tx.len;
  const int lim_lo = a.causal ? max(r0 + 1, tx.prefix) : tx.len, lim_hi = a.causal ? max(r0 + 32, tx.prefix) : tx.len;
  const uint8_t* mask = a.mask ? a.mask + tx.m0 : nullptr;
  const bool terms = a.bias || a.slope;
  const float slope = a.slope ? a.slope[p.h] : 0.f;
  const float qs = a.scale * (a.cap > 0.f ? 1.f / a.cap : LOG2E), c_out = a.cap * LOG2E;

  f32x4 qf[NI];
  {
    const float* Q = (const float*)a.q + tx.q0 + (long)r * a.q_ld + p.h * a.q_head;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int c = 8 * i + 4 * lh;
      qf[i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (r < tx.len && c < d) qf[i] = *(const f32x4*)(Q + c);
    }
  }
  f32x16 o[ND];
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  float m_run = -INFINITY, l = 0.f;
  if (tid < 3) odd[tid] = 0;
  __syncthreads();

  const float* K = (const float*)a.k + tx.k0 + p.g * a.k_head;
  const float* V = (const float*)a.v + tx.v0 + p.g * a.v_head;
  f32x4 rk[CPT], rv[CPT];
  float rb = 0.f;
  auto far_of = [&](int k0) { return k0 - b0 + min(tid, KT + TQ - 2) - (TQ - 1); };
  auto fetch = [&](int k0, uint32_t bits) __attribute__((always_inline)) {
    const int n = min(KT, k_end - k0);
    const __amdgpu_buffer_rsrc_t kr = make_rsrc(K + (long)k0 * a.k_ld, ((n - 1) * (long)a.k_ld + d) * 4);
    const __amdgpu_buffer_rsrc_t vr = make_rsrc(V + (long)k0 * a.v_ld, ((n - 1) * (long)a.v_ld + d) * 4);
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const int idx = tid + NT * i, key = idx / (D32 / 4), c = idx % (D32 / 4) * 4;
      const bool on = (bits >> key & 1) && c < d;
      rk[i] = __builtin_bit_cast(f32x4, buf_load16(kr, on ? (key * (int)a.k_ld + c) * 4 : OOB));
      rv[i] = __builtin_bit_cast(f32x4, buf_load16(vr, on ? (key * (int)a.v_ld + c) * 4 : OOB));
    }
    if (terms) rb = table_at(a, p.h, far_of(k0));  // (and `stage` makes the term of it, behind the products)
  };
  auto stage = [&](int b, int k0, int slot) __attribute__((always_inline)) {
    const bool border = a.causal && k0 + KT > max(b0 + 1, tx.prefix);
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
      const int idx = tid + NT * i, key = idx / (D32 / 4), c = idx % (D32 / 4) * 4;
      *(f32x4*)&Ks[b][key * LDK + c] = rk[i];
      f32x4 v = rv[i];
      if (border)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (odd_f(v[e])) {
            odd[slot] = 1;
            v[e] = 0.f;
          }
      *(f32x4*)&Vs[b][key * LDV + c] = v;
    }
    if (terms && tid < KT + TQ - 1) strip[b][tid] = term_of(rb, far_of(k0), slope, 1.f);
  };
  const __amdgpu_buffer_rsrc_t mr = make_rsrc(mask, k_end);
  auto own_mask = [&](int k0) -> int { return mask ? (int)__builtin_amdgcn_raw_buffer_load_b8(mr, k0 + lq, 0, 0) : 1; };
  auto ballot = [&](int k0, int own) -> uint32_t { return (uint32_t)__ballot(k0 + lq < k_end && own); };
  const int sb = TQ - 1 - wave * 32 - lq + 4 * lh;
  if (k_end > 0) {
    int own = own_mask(0);
    uint32_t bits = ballot(0, own);
    own = own_mask(KT);
    fetch(0, bits);
    stage(0, 0, 0);
    __syncthreads();
    for (int k0 = 0, b = 0, slot = 0; k0 < k_end; k0 += KT, b ^= 1) {
      uint32_t next = 0;
      const bool more = k0 + KT < k_end;
      if (more) {
        next = ballot(k0 + KT, own);
        own = own_mask(k0 + 2 * KT);
        fetch(k0 + KT, next);
      }
      const int s1 = slot == 2 ? 0 : slot + 1;
      if (bits && k0 < lim_hi && r0 < tx.len) {
        // (fragments ahead of their products where registers allow; channels from d on are
        // zeros; two sums, so that each is half as long a chain of roundings)
        f32x16 s = {}, s2 = {};
        constexpr int AHEAD = D32 <= 128 ? NI : 4;
#pragma unroll
        for (int i0 = 0; i0 < NI; i0 += AHEAD) {
          f32x4 kf[AHEAD];
#pragma unroll
          for (int i = 0; i < AHEAD; ++i) kf[i] = *(const f32x4*)&Ks[b][lq * LDK + 8 * (i0 + i) + 4 * lh];
#pragma unroll
          for (int i = 0; i < AHEAD; ++i)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
              s = mfma_f32(kf[i][e], qf[i0 + i][e], s);
              s2 = mfma_f32(kf[i][e + 1], qf[i0 + i][e + 1], s2);
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = (s[i] + s2[i]) * qs;
        // register i: key 8 (i / 4) + 4 lh + i % 4
        if (a.cap > 0.f)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = c_out * tanh_f32(s[i]);
        if (terms)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] += strip[b][sb + 8 * (i >> 2) + (i & 3)];
        if (bits != ~0u || k0 + KT > lim_lo) {
          const uint32_t bm = bits >> (4 * lh);
          const int left = lim - k0 - 4 * lh;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int c = 8 * (i >> 2) + (i & 3);
            if (c >= left || !(bm >> c & 1)) s[i] = -INFINITY;
          }
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
        // (a tile's sums are made apart and added: over the keys one after another, a long
        // text's roundings would add up)
        float lt = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[i] = __builtin_amdgcn_exp2f(s[i] - ref);
          lt += s[i];
        }
        l += lt;
#pragma unroll
        for (int t = 0; t < ND; ++t) {
          f32x16 ot = {};
#pragma unroll
          for (int i = 0; i < 16; ++i) ot = mfma_f32(Vs[b][(8 * (i >> 2) + 4 * lh + (i & 3)) * LDV + lq + 32 * t], s[i], ot);
#pragma unroll
          for (int i = 0; i < 16; ++i) o[t][i] += ot[i];
        }
        if (a.causal && odd[slot]) {
#pragma unroll 1
          for (int j = 0; j < KT; ++j) {
            if (!(bits >> j & 1)) continue;
            const __amdgpu_buffer_rsrc_t vr = make_rsrc(V + (long)(k0 + j) * a.v_ld, d * 4);
            const bool seen = k0 + j < lim;
#pragma unroll
            for (int t = 0; t < ND; ++t)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const f32x4 x = __builtin_bit_cast(f32x4, buf_load16(vr, (32 * t + 8 * i + 4 * lh) * 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) o[t][4 * i + e] += seen && odd_f(x[e]) ? x[e] : 0.f;
              }
          }
        }
      }
      if (more) stage(b ^ 1, k0 + KT, s1);
      if (tid == 0) odd[s1 == 2 ? 0 : s1 + 1] = 0;
      __syncthreads();
      bits = next;
      slot = s1;
    }
  }
  const float2 hl = half_swap(l);
  l = hl.x + hl.y;
  if (r >= rows) return;
  float* out = (float*)a.o + tx.o0 + (long)r * a.o_ld + p.h * a.o_head;
  const float f = l == 0.f ? 0.f : 1.0f / l;
  const bool live = r < tx.len;
#pragma unroll
  for (int t = 0; t < ND; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = 32 * t + 8 * i + 4 * lh;
      if (c < d) {
        f32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = live ? o[t][4 * i + e] * f : 0.f;
        *(f32x4*)(out + c) = w;
      }
    }
}

// ------------------------------------------------------------------ launch
template <int D16, bool SHORT>
static void launch_kind(const TextArgs& a, dim3 grid, hipStream_t s) {
  const bool terms = a.bias || a.slope;
  if (a.cap > 0.f) {
    if (terms) text_bf16_kernel<D16, true, true, SHORT><<<grid, 256, 0, s>>>(a);
    else text_bf16_kernel<D16, false, true, SHORT><<<grid, 256, 0, s>>>(a);
  } else {
    if (terms) text_bf16_kernel<D16, true, false, SHORT><<<grid, 256, 0, s>>>(a);
    else text_bf16_kernel<D16, false, false, SHORT><<<grid, 256, 0, s>>>(a);
  }
}
template <int D16>
static void launch_width(const TextArgs& a, dim3 grid, hipStream_t s) {
  // (both sides measured: see the kernel)
  if (a.max_len <= 128) launch_kind<D16, true>(a, grid, s);
  else launch_kind<D16, false>(a, grid, s);
}

// The grid of a call (x = 0 past its limits), and how it is dealt (a.chunk, a.chunks).
static dim3 grid_of(TextArgs& a) {
  const long tiles = a.max_len < 1 ? 1 : ((long)a.max_len + TQ - 1) / TQ;  // (packed rows of no text may still be due zeros)
  a.chunk = (int)(tiles < 8 ? tiles : 8);  // (1, 8, 32: 16 x 512 tokens, 20 heads of 64 39.3, 36.3, 37.4 us; 4 x 4000 426, 406, 402)
  a.chunks = (int)((tiles + a.chunk - 1) / a.chunk);
  const long y = ((long)a.n * a.kv_heads + 7) / 8, x = 8L * a.chunk * a.rep;
  if (y > 65535 || a.chunks > 65535 || (double)x * y * a.chunks * 256 > 4.0e9) return dim3(0);
  return dim3((unsigned)x, (unsigned)y, (unsigned)a.chunks);
}

bool text_attention_fits(int n, int heads, int kv_heads, int max_len) {
  TextArgs a;
  a.n = n; a.kv_heads = kv_heads; a.rep = heads / kv_heads; a.max_len = max_len;
  return grid_of(a).x > 0;
}

hipError_t launch_text_attention(DType dt, TextArgs a, hipStream_t s) {
  if (a.n <= 0) return hipSuccess;
  const dim3 grid = grid_of(a);
  if (grid.x == 0) return hipErrorInvalidValue;
  if (dt == BF16) {
    if (a.d <= 32) launch_width<32>(a, grid, s);
    else if (a.d <= 48) launch_width<48>(a, grid, s);
    else if (a.d <= 64) launch_width<64>(a, grid, s);
    else if (a.d <= 80) launch_width<80>(a, grid, s);
    else if (a.d <= 96) launch_width<96>(a, grid, s);
    else if (a.d <= 128) launch_width<128>(a, grid, s);
    else if (a.d <= 192) launch_width<192>(a, grid, s);
    else launch_width<256>(a, grid, s);
  } else {
    if (a.d <= 32) text_f32_kernel<32><<<grid, 256, 0, s>>>(a);
    else if (a.d <= 64) text_f32_kernel<64><<<grid, 256, 0, s>>>(a);
    else if (a.d <= 96) text_f32_kernel<96><<<grid, 256, 0, s>>>(a);
    else if (a.d <= 128) text_f32_kernel<128><<<grid, 256, 0, s>>>(a);
    else if (a.d <= 192) text_f32_kernel<192><<<grid, 256, 0, s>>>(a);
    else text_f32_kernel<256><<<grid, 256, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace sd
