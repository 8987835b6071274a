// Attention by tiles of 128 query rows: kernel and launch, instantiated by mt_mha_tile_*.hip.
#pragma once

#include "mt_mha_dev.h"

namespace mt {

typedef float f32x16 __attribute__((ext_vector_type(16)));

// The two element types' MFMAs of 32 keys (rows) by 32 queries (columns).  An operand's lane holds row or column
// lane % 32; a result's lane holds column lane % 32 and rows 8 (r / 4) + 4 (lane / 32) + r % 4.  Which depth a lane's
// elements stand for is free as long as both operands agree: the weights P of a tile leave the first product with
// a lane's keys 4 (lane / 32) + .. of every eight, and are taken for the second one in just that order.
template <typename T>
struct Tile;

template <>
struct Tile<bf16> {
  static constexpr int KT = 64;    // keys of a tile
  static constexpr int STEP = 16;  // features of a step of q.k
  typedef bf16x8 Q;                // features 16 s + 8 (lane / 32) + ..
  // the 64 banks take 16 rows' chunks of keys at a time, or 4 rows' chunks of 32 neighbouring features (values,
  // transposed): the chunks of 16 bytes of a row are permuted by its number so that they fall into different banks
  template <int ROWB>
  __device__ static __forceinline__ int swap_v(int row) {
    return ROWB >= 256 ? (row & 3) << 2 : (row & 2) << 1;
  }
  // Of two elements (one in fp32) those that are no numbers: infinities go to plus as 2^127 or to minus as -2^127, NaN to both, whose
  // products with 2^127 are infinities again and with zero nothing.  Gives the elements that are numbers.
  __device__ static __forceinline__ unsigned split(unsigned v, unsigned &plus, unsigned &minus) {
    auto all = [](unsigned bits) { return (bits & 0x00010001u) * 0xffffu; };
    const unsigned over = all(((v & 0x7f807f80u) + 0x00800080u) >> 15), nan = all(((v & 0x007f007fu) + 0x007f007fu) >> 7) & over;
    const unsigned below = all(v >> 15);
    plus = over & (nan | ~below) & 0x7f007f00u;
    minus = over & (nan | below) & 0xff00ff00u;
    return v & ~over;
  }
  __device__ static __forceinline__ void qk(f32x16 &s, const char *k, const Q &q) {
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8 *)k, q, s, 0, 0, 0);
  }
};

template <>
struct Tile<float> {
  static constexpr int KT = 32;
  static constexpr int STEP = 8;
  typedef f32x4 Q;  // features 8 s + 4 (lane / 32) + ..
  // values: 32 neighbouring features of two rows four apart
  template <int ROWB>
  __device__ static __forceinline__ int swap_v(int row) {
    return (row & 4) << 1;
  }
  __device__ static __forceinline__ unsigned split(unsigned v, unsigned &plus, unsigned &minus) {
    const bool over = (v & 0x7f800000u) == 0x7f800000u, nan = over && (v & 0x007fffffu), below = v >> 31;
    plus = over && (nan || !below) ? 0x7f000000u : 0u;
    minus = over && (nan || below) ? 0xff000000u : 0u;
    return over ? 0u : v;
  }
  __device__ static __forceinline__ void qk(f32x16 &s, const char *k, const Q &q) {
    const f32x4 kk = *(const f32x4 *)k;
#pragma unroll
    for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(kk[e], q[e], s, 0, 0, 0);
  }
};

template <int ROWB>
__device__ __forceinline__ int swap_k(int row) {
  return ROWB >= 256 ? row & 15 : (row >> 1) & 7;
}

__device__ __forceinline__ float both_halves_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return fmaxf(__int_as_float(r[0]), __int_as_float(r[1]));
}
__device__ __forceinline__ float both_halves_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(v), __float_as_int(v), false, false);
  return __int_as_float(r[0]) + __int_as_float(r[1]);
}

// Sets bits of `over` where one of the elements of v is an infinity or a NaN: an exponent of all ones passes into the
// sign's place when one is added.
template <typename T>
__device__ __forceinline__ void note_nonfinite(const int4 &v, unsigned &over) {
  constexpr unsigned field = sizeof(T) == 2 ? 0x7f807f80u : 0x7f800000u, one = sizeof(T) == 2 ? 0x00800080u : 0x00800000u;
  over |= ((unsigned)v.x & field) + one;
  over |= ((unsigned)v.y & field) + one;
  over |= ((unsigned)v.z & field) + one;
  over |= ((unsigned)v.w & field) + one;
}
template <typename T>
__device__ __forceinline__ bool nonfinite(unsigned over) {
  return over & (sizeof(T) == 2 ? 0x80008000u : 0x80000000u);
}

// One wave's 32 queries, a query per lane (and half of a tile's keys): its features, and the running softmax.
template <typename T, int DP>
struct Rows {
  typedef Tile<T> M;
  static constexpr int ES = sizeof(T), STEPS = DP / M::STEP, DB = DP / 32, ROWB = DP * ES;
  typename M::Q q[STEPS];
  f32x16 o[DB];  // features 32 d + 8 (r / 4) + 4 (lane / 32) + r % 4
  float m, l;    // maximum that the sums are relative to; this half's sum of weights
  float bound;   // the score from which the maximum moves (wide heads have no register for it)

  __device__ __forceinline__ void start(const T *src, bool live, int Dh) {
    constexpr int VEC = 16 / ES;
    const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int d = s * M::STEP + half * VEC;
      typename Vec<T, VEC>::Raw v = {};
      if (live && d < Dh) v = Vec<T, VEC>::raw_any(src + d);
      __builtin_memcpy(&q[s], &v, 16);
    }
    clear();
    m = bound = kNegInf;
    l = 0.f;
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = (f32x16)(0.f);
  }

  // scores of 32 keys, rows row0 .. of the tile in LDS
  __device__ __forceinline__ f32x16 scores(const char *keys, int row0) const {
    f32x16 s = (f32x16)(0.f);
    const int lane = threadIdx.x & 63, row = row0 + (lane & 31), half = lane >> 5;
#pragma unroll
    for (int st = 0; st < STEPS; ++st) M::qk(s, keys + row * ROWB + (((2 * st + half) ^ swap_k<ROWB>(row)) << 4), q[st]);
    return s;
  }

  // Weights relative to a maximum that only moves where a score passes it by 2^8: the sums stay far inside 32 bits,
  // and the accumulators are rescaled a few times in a row's life.
  template <int KB>
  __device__ __forceinline__ void weights(f32x16 (&s)[KB], float scale) {
    float mx = kNegInf;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[kb][e]);
    mx = both_halves_max(mx) * scale;
    float use = m == kNegInf ? 0.f : m;
    if (__builtin_expect(__any(mx > (DP > 128 ? max_bound(m) : bound)), 0)) {
      const float mn = fmaxf(m, mx), c = m == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      bound = max_bound(m);
      use = m == kNegInf ? 0.f : m;
      l *= c;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] *= c;
      const bool far = fabsf(use) >= kFarScore;
      if (__builtin_expect(__any(far), 0)) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            s[kb][e] = far ? rounded_product(s[kb][e], scale) - use : fmaf(s[kb][e], scale, -use);
        scale = 1.f;  // the exponents as they are
        use = 0.f;
      }
    }
    float sum[2] = {};
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[kb][e] = __builtin_amdgcn_exp2f(fmaf(s[kb][e], scale, -use));
        sum[e & 1] += s[kb][e];
      }
    l += sum[0] + sum[1];
  }

  // The products of 32 keys' weights with their values, rows row0 .. of the tile in LDS.  In bf16 the weights are rounded to the
  // values' type, 2^-8 each at most, for one product of the matrix units: results are as far from exact as their own rounding makes
  // them, so 1.4 times as far together (2.3e-3 of a norm, where the row kernel's have 1.7e-3).  With the weights' rest as a
  // second product they are not, and take longer: 2 x 2048 positions over 8192, 32 heads of 128, 524 -> 688 us, 8 ragged sentences
  // of up to 2048 x 2048 of 16 heads of 64 82 -> 105, 16 tokens over 32768 369 -> 371, 30 tokens of a window of 5 6.9 -> 7.1.
  __device__ __forceinline__ void values(const char *vals, int row0, const f32x16 &s) {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    if constexpr (ES == 2) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef s16x4 __attribute__((address_space(3))) * Lp;
      const int l16 = lane & 15;
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        bf16x8 p;
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (bf16)s[hf * 8 + e];
        const int row = row0 + hf * 16 + 4 * half + l16 / 4;
        const char *from = vals + row * ROWB + (l16 & 1) * 8;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const int c = (4 * d + 2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1)) ^ M::template swap_v<ROWB>(row);
          union {
            s16x4 q[2];
            bf16x8 v;
          } f;
          // a lane's 8 bytes go to four lanes: it receives one feature of four keys
          f.q[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lp)(from + (c << 4)));
          f.q[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lp)(from + 8 * ROWB + (c << 4)));
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v, p, o[d], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int row = row0 + 8 * (e / 4) + 4 * half + e % 4;
#pragma unroll
        for (int d = 0; d < DB; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(
              *(const float *)(vals + row * ROWB + (((d * 32 + (lane & 31)) * 4) ^ (M::template swap_v<ROWB>(row) << 4))), s[e], o[d], 0,
              0, 0);
      }
    }
  }

  // What values that are no numbers make of the sums of the queries that see them, where the tile's products had zeros for them:
  // infinities and NaN, added to o.  32 keys, rows row0 .. of the tile in LDS as it was in memory; a query sees this lane's key i of
  // them where first + i < n.  Products of one sign overflow by themselves; together with the others', or added to an infinity by
  // the product, they would not.
  __device__ __forceinline__ void odd_values(const char *vals, int row0, unsigned first, unsigned n) {
    const int lane = threadIdx.x & 63, half = lane >> 5;
    auto seen = [&](int e) { return first + 8 * (e / 4) + e % 4 < n ? 0x1p127f : 0.f; };
    if constexpr (ES == 2) {
      typedef short s16x4 __attribute__((ext_vector_type(4)));
      typedef s16x4 __attribute__((address_space(3))) * Lp;
      const int l16 = lane & 15;
#pragma unroll 1
      for (int hf = 0; hf < 2; ++hf) {
        bf16x8 p;
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = (bf16)seen(hf * 8 + e);
        const int row = row0 + hf * 16 + 4 * half + l16 / 4;
        const char *from = vals + row * ROWB + (l16 & 1) * 8;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const int c = (4 * d + 2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1)) ^ M::template swap_v<ROWB>(row);
          union {
            s16x4 q[2];
            unsigned w[4];
            bf16x8 v;
          } f, minus;
          f.q[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lp)(from + (c << 4)));
          f.q[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lp)(from + 8 * ROWB + (c << 4)));
#pragma unroll
          for (int i = 0; i < 4; ++i) M::split(f.w[i], f.w[i], minus.w[i]);
          o[d] += __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v, p, (f32x16)(0.f), 0, 0, 0);
          o[d] += __builtin_amdgcn_mfma_f32_32x32x16_bf16(minus.v, p, (f32x16)(0.f), 0, 0, 0);
        }
      }
    } else {
#pragma unroll 1
      for (int e = 0; e < 16; ++e) {
        const int row = row0 + 8 * (e / 4) + 4 * half + e % 4;
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          unsigned plus, minus;
          M::split(*(const unsigned *)(vals + row * ROWB + (((d * 32 + (lane & 31)) * 4) ^ (M::template swap_v<ROWB>(row) << 4))), plus, minus);
          o[d] += __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(plus), seen(e), (f32x16)(0.f), 0, 0, 0);
          o[d] += __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(minus), seen(e), (f32x16)(0.f), 0, 0, 0);
        }
      }
    }
  }

  // adds o to what put or put_part has stored
  template <typename R>
  __device__ __forceinline__ void add(R *y, int Dh) const {
    const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int f = d * 32 + 2 * e + 4 * half;
        if (f >= Dh) continue;
        const auto was = Vec<R, 4>::raw_any(y + f);
        const float v[4] = {(float)was.v[0] + o[d][e], (float)was.v[1] + o[d][e + 1], (float)was.v[2] + o[d][e + 2], (float)was.v[3] + o[d][e + 3]};
        Vec<R, 4>::put_any(y + f, v);
      }
  }

  // sums and their pair of a part (l: of both halves)
  __device__ __forceinline__ void put_part(float *po, float2 *pml, int Dh) const {
    const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int f = d * 32 + 2 * e + 4 * half;
        if (f < Dh) *(float4 *)(po + f) = make_float4(o[d][e], o[d][e + 1], o[d][e + 2], o[d][e + 3]);
      }
    if (half == 0) *pml = make_float2(m, l);
  }
  __device__ __forceinline__ void put(T *y, int Dh) const {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const int f = d * 32 + 2 * e + 4 * half;
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = times_or_zero(o[d][e + i], inv);
        if (f < Dh) Vec<T, 4>::put_any(y + f, v);
      }
  }
};

// scores of keys that a query does not see: of 32 keys from k0 on, those outside [lo, hi) or whose bit of seen is 0
template <bool PAGED>
__device__ __forceinline__ void hide(f32x16 &s, int k0, int lo, int hi, unsigned seen) {
  int first = 4 * ((threadIdx.x >> 5) & 1);
  asm volatile("" : "+v"(first));  // a branch: without it the selects move into every tile
  const unsigned from = k0 + first - lo, n = max(hi - lo, 0), bits = seen >> first;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int kk = 8 * (e / 4) + e % 4;
    s[e] = (PAGED ? from + kk < n : (bits >> kk) & 1) ? s[e] : kNegInf;
  }
}

constexpr int kTileRows = 128;

// Brings tiles of KT keys and values from memory to LDS by TH threads: a tile's chunks of 16 bytes are on their way in
// registers while the one before is computed, and its page numbers (mask) a tile earlier still.  A wave's 64 chunks are at
// most eight neighbouring rows, beginning at a multiple of their number, so they lie in one page: page numbers and
// bases are the wave's, and what a lane adds to them is the same in every tile.
template <typename T, int DP, bool PAGED, int KT, int TH>
struct Mover {
  typedef Tile<T> M;
  static constexpr int ES = sizeof(T), CH = DP * ES / 16, ROWB = DP * ES, TB = KT * ROWB;
  static constexpr int NL = KT * CH / TH, RSTEP = TH / CH;  // chunks of a thread, all of one column
  static_assert(TH % CH == 0 && KT % RSTEP == 0 && 64 % CH == 0 && 64 / CH <= 8, "a wave's rows lie in one page");
  const char *k, *v;        // of this key head (and sequence)
  long long ldk, ldv;       // not paged: bytes of a row
  long long lane_k, lane_v; // not paged: this lane's bytes from its wave's first row
  unsigned lane_at;         // paged: the same
  unsigned page_bytes;
  const int32_t *table;
  const float *mask;
  int row, chunk, wave_row, last, plog, top, rowb;
  bool feature;             // whether the column is one of the head's
  int bad;                  // not 0: a page number was out of range
  int pg[NL];
  float valid;              // mask of key lane of the next tile
  unsigned long long seen;  // keys of the tile on its way that are there and not masked
  int4 kr[NL], vr[NL];

  __device__ __forceinline__ void start(const MhaArgs &a, int b, int h, int tid, int last_key, const float *m) {
    row = tid / CH;
    chunk = tid % CH;
    wave_row = TH == 64 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6) * (64 / CH);
    feature = chunk * 16 < a.Dh * ES;
    last = last_key;
    plog = a.page_log2;
    top = a.n_pages - 1;
    rowb = a.Dh * ES;
    bad = 0;
    mask = m;
    seen = 0;
    const int col = feature ? chunk * 16 : 0;  // columns that only pad read the first one and become zeros
    if (PAGED) {
      table = a.table + (long long)b * a.n_blocks;
      page_bytes = ((unsigned)a.Hk << plog) * rowb;
      const long long at = ((long long)h << plog) * rowb;
      k = (const char *)a.k + at;
      v = (const char *)a.v + at;
      lane_at = (row - wave_row) * rowb + col;
    } else {
      ldk = a.ldk * ES;
      ldv = a.ldv * ES;
      k = (const char *)a.k + (long long)b * a.Sk * ldk + h * rowb;
      v = (const char *)a.v + (long long)b * a.Sk * ldv + h * rowb;
      lane_k = (row - wave_row) * ldk + col;
      lane_v = (row - wave_row) * ldv + col;
    }
  }
  // what a tile's loads will need; blocks behind the last key stand for its own
  __device__ __forceinline__ void look(int k0) {
    if (PAGED) {
#pragma unroll
      for (int x = 0; x < NL; ++x) pg[x] = table[min(k0 + wave_row + x * RSTEP, last) >> plog];
    } else if (mask) {
      valid = mask[min(k0 + (int)(threadIdx.x & 63), last)];
    }
  }
  // ahead: keys to the tile after it
  __device__ __forceinline__ void fetch(int k0, int ahead) {
    if (PAGED) {
      // positions behind the last key are read too, inside its page; put makes zeros of their values
      const int pmask = (1 << plog) - 1;
#pragma unroll
      for (int x = 0; x < NL; ++x) {
        const int page = min(max(pg[x], 0), top);
        bad |= page ^ pg[x];
        const unsigned long long at = (unsigned long long)(unsigned)page * page_bytes + (unsigned)((k0 + wave_row + x * RSTEP) & pmask) * rowb;
        kr[x] = *(const int4 *)(k + at + lane_at);
        vr[x] = *(const int4 *)(v + at + lane_at);
      }
    } else {
      const int j = threadIdx.x & 63;
      seen = __ballot(j < KT && k0 + j <= last && (!mask || valid != 0.f));
      if (k0 + KT - 1 <= last) {
#pragma unroll
        for (int x = 0; x < NL; ++x) load_rows(x, (k0 + wave_row + x * RSTEP) * ldk + lane_k, (k0 + wave_row + x * RSTEP) * ldv + lane_v);
      } else {  // rows behind the last key stand for it
#pragma unroll
        for (int x = 0; x < NL; ++x) {
          const long long back = min(0, last - (k0 + row + x * RSTEP));
          load_rows(x, (k0 + wave_row + x * RSTEP + back) * ldk + lane_k, (k0 + wave_row + x * RSTEP + back) * ldv + lane_v);
        }
      }
    }
    look(k0 + ahead);
  }
  __device__ __forceinline__ void load_rows(int x, long long ak, long long av) {
    const auto kv = Vec<T, 16 / ES>::raw_any((const T *)(k + ak)), vv = Vec<T, 16 / ES>::raw_any((const T *)(v + av));
    __builtin_memcpy(&kr[x], &kv, 16);
    __builtin_memcpy(&vr[x], &vv, 16);
  }
  // The tile that was fetched, into LDS.  Values that no row may see are zeros (their weights are).  mixed: some rows see
  // keys of the tile that others do not; values that are no numbers, which zeros of weights would not hide, are zeros then, and
  // said to have been there.
  __device__ __forceinline__ bool put(int k0, char *buf, bool mixed) {
    unsigned over = 0;
    const bool all = PAGED ? k0 + KT - 1 <= last : seen == (KT == 64 ? ~0ull : (1ull << KT) - 1);
    if (!all || rowb != ROWB) {
#pragma unroll
      for (int x = 0; x < NL; ++x) {
        const int r = row + x * RSTEP;
        const bool there = feature && (PAGED ? k0 + r <= last : (seen >> r) & 1);
        if (!feature) kr[x] = make_int4(0, 0, 0, 0);
        if (!there) vr[x] = make_int4(0, 0, 0, 0);
      }
    }
    if (PAGED && mixed) {
#pragma unroll
      for (int x = 0; x < NL; ++x) note_nonfinite<T>(vr[x], over);
    }
#pragma unroll
    for (int x = 0; x < NL; ++x) {
      const int r = row + x * RSTEP;
      *(int4 *)(buf + r * ROWB + ((chunk ^ swap_k<ROWB>(r)) << 4)) = kr[x];
      *(int4 *)(buf + TB + r * ROWB + ((chunk ^ M::template swap_v<ROWB>(r)) << 4)) = vr[x];
    }
    const bool odd = nonfinite<T>(over);
    if (PAGED && __builtin_expect(odd, 0)) {
#pragma unroll 1
      for (int r = row; r < KT; r += RSTEP) {
        int4 *const at = (int4 *)(buf + TB + r * ROWB + ((chunk ^ M::template swap_v<ROWB>(r)) << 4)), v = *at;
        unsigned a, b;
        *at = make_int4(M::split(v.x, a, b), M::split(v.y, a, b), M::split(v.z, a, b), M::split(v.w, a, b));
      }
    }
    return odd;
  }
  // The values of a tile once more, as they are in memory (few registers: what it follows needs them)
  __device__ __forceinline__ void put_again(int k0, char *buf) const {
#pragma unroll 1
    for (int x = 0; x < KT; x += RSTEP) {
      const int r = row + x, j = k0 + wave_row + x, page = min(max(table[min(j, last) >> plog], 0), top);
      const unsigned long long at = (unsigned long long)(unsigned)page * page_bytes + (unsigned)(j & ((1 << plog) - 1)) * rowb;
      int4 w = *(const int4 *)(v + at + lane_at);
      if (!feature || k0 + r > last) w = make_int4(0, 0, 0, 0);
      *(int4 *)(buf + TB + r * ROWB + ((chunk ^ M::template swap_v<ROWB>(r)) << 4)) = w;
    }
  }
};

// What a launch of the tile kernel has decided
struct TilePlan {
  int tiles;  // of kTileRows rows of a sequence's key head
  int parts;  // the key axis is cut into
  int first;  // workgroup of this launch
  bool fold;  // whether a row's tiles differ much in their keys
  const int *order;   // masked sentences, those with the most work first, or NULL: as they come
  const int2 *edges;  // of each sentence's mask: its first valid position, one past its last; or NULL: not yet known
};

// A workgroup of four waves takes 128 rows of one key head of one sequence: row r is query r / G, head r % G of those
// that share the key head.  Keys and values pass through LDS a tile at a time, the next tile's on their way in registers
// while this one's is computed.  Scores transposed: S = K Q^T has a query per lane and its keys in registers, so the
// softmax needs one exchange between a wave's halves, and P^T is the second product's operand as it stands.
// 2 x 2048 positions over 8192, 32 heads of 128 (8 of keys) in bf16: 518 us, 929 TFLOP/s where a large product reaches 1192.
// LDS is active in 59% of the cycles, vector and matrix units in 40% each: a unit's two waves are in step, and more waves do
// not fit their registers.  With conflicts between LDS banks it took 574 us, with masks in every tile 883.
template <typename T, int DP, bool PAGED>
__global__ void __launch_bounds__(256, DP <= 128 ? 2 : 1) tile_kernel(MhaArgs a, TilePlan plan) {
  typedef Tile<T> M;
  // heads of more than 128 features leave no registers for more keys at a time; in fp32 some 70 are spilled all the same
  constexpr int KT = DP > 128 ? 32 : M::KT, TB = KT * DP * (int)sizeof(T), KB = KT / 32;
  __shared__ __attribute__((aligned(1024))) char lds[4 * TB];
  __shared__ int dirty, edge[2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31;
  // the tiles of a key head run on one XCD, whose L2 holds its keys and values, the heads of a sequence on different
  // ones; what does not divide among them is spread.  The last tiles, which see the most keys, come first.
  const int w = plan.first + blockIdx.x, per = plan.tiles * plan.parts, heads = a.B * a.Hk, even = heads / kXcds * kXcds;
  // Where all workgroups run at once, two a unit, and the first rows see few keys: the second of a unit is taken from the
  // other end, a short one with a long one (4 x 1000 positions of 16 heads of 64: fp32 144 -> 97 us, bf16 28 -> 24).
  auto fold = [&](int v, int n, int units) { return plan.fold && v >= units && n <= 2 * units ? units + n - 1 - v : v; };
  int bh, u;
  if (w < even * per) {
    const int v = fold(w / kXcds, even / kXcds * per, a.num_cu / kXcds);
    const int round = v / per, x = w % kXcds;
    bh = round * kXcds + (plan.order && round % 2 ? kXcds - 1 - x : x);  // sorted by work: there and back
    u = v % per;
  } else {
    const int v = fold(w - even * per, (heads - even) * per, a.num_cu);
    bh = even + v / per;
    u = v % per;
  }
  const int part = u % plan.parts, tile = plan.tiles - 1 - u / plan.parts;
  const int place = bh / a.Hk, h = bh - place * a.Hk, b = plan.order ? plan.order[place] : place;
  const RowSpan span = row_span<PAGED>(a, b, h == 0 && tile == 0 && part == 0 && threadIdx.x == 0);
  const int R = span.n * a.G, r0 = tile * kTileRows;
  if (r0 >= R) return;
  const int i_first = r0 / a.G, i_last = min(r0 + kTileRows - 1, R - 1) / a.G;
  int lo, hi, lo2, hi2;  // keys that some row sees: [lo, hi2); that all see: [lo2, hi)
  seen_keys<PAGED>(a, span, i_first, lo, hi);
  seen_keys<PAGED>(a, span, i_last, lo2, hi2);
  if (threadIdx.x == 0) dirty = 0;
  const float *mask = !PAGED && a.mask ? a.mask + (long long)b * a.Sk : nullptr;
  if (!PAGED && mask && plan.edges) {
    const int2 e = plan.edges[b];
    lo = e.x;
    hi2 = e.y;
  } else if (!PAGED && mask) {  // the first and the last valid position
    if (threadIdx.x == 0) edge[0] = a.Sk, edge[1] = 0;
    __syncthreads();
    int first, last;
    mask_ends<4>(mask, a.Sk, threadIdx.x, 256, first, last);
    if (last) atomicMin(&edge[0], first), atomicMax(&edge[1], last);
    __syncthreads();
    lo = edge[0];
    hi2 = edge[1];
  }
  if (PAGED) __syncthreads();  // dirty is set from here on
  lo &= ~(KT - 1);
  int nt = hi2 > lo ? (hi2 - lo + KT - 1) / KT : 0;  // tiles of keys, this part's of them
  {
    const int per = (nt + plan.parts - 1) / plan.parts;
    const int t0 = min(nt, part * per);
    nt = min(nt, t0 + per) - t0;
    lo += t0 * KT;
  }
  // ---- this lane's query
  const int r = r0 + wave * 32 + col;
  const bool live = r < R;
  const int qi = (live ? r : R - 1) / a.G, hq = h * a.G + (live ? r : R - 1) - qi * a.G;
  int qlo, qhi;
  seen_keys<PAGED>(a, span, qi, qlo, qhi);
  Rows<T, DP> me;
  me.start((const T *)a.q + ((long long)b * a.S + qi) * a.ldq + (long long)hq * a.Dh, live, a.Dh);
  // keys that some row of this wave sees
  int wlo = 0, whi = 0;
  {
    const int first = r0 + wave * 32, last = min(first + 31, R - 1);
    int x;
    if (first < R) seen_keys<PAGED>(a, span, first / a.G, wlo, x), seen_keys<PAGED>(a, span, last / a.G, x, whi);
  }
  // ---- tiles of keys
  Mover<T, DP, PAGED, KT, 256> mv;
  auto mixed = [&](int k0) { return k0 + KT > hi || k0 < lo2; };
  if (nt > 0) {
    mv.start(a, b, h, threadIdx.x, hi2 - 1, mask);
    mv.look(lo);
    mv.fetch(lo, KT);
    if (mv.put(lo, lds, mixed(lo))) dirty = 1;
  }
  for (int t = 0; t < nt; ++t) {
    const int k0 = lo + t * KT;
    const char *buf = lds + (t & 1) * 2 * TB;
    const unsigned long long seen = mv.seen;
    __syncthreads();
    if (t + 1 < nt) mv.fetch(k0 + KT, KT);
    if (k0 < whi && k0 + KT > wlo) {
      f32x16 s[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[kb] = me.scores(buf, kb * 32);
      if (PAGED ? mixed(k0) : seen != (KT == 64 ? ~0ull : (1ull << KT) - 1)) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) hide<PAGED>(s[kb], k0 + kb * 32, qlo, qhi, (unsigned)(seen >> (kb * 32)));
      }
      me.weights(s, a.scale);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) me.values(buf + TB, kb * 32, s[kb]);
    }
    if (t + 1 < nt && mv.put(k0 + KT, lds + ((t + 1) & 1) * 2 * TB, mixed(k0 + KT))) dirty = 1;
  }
  if (PAGED && nt > 0 && mv.bad) atomicOr(a.err, kErrPage);
  // ---- results
  me.l = both_halves_sum(me.l);
  const long long rows = (long long)a.B * a.Hq * a.S;
  const Parts parts = parts_of(a.ws, rows, plan.parts);
  const long long prow = part * rows + ((long long)b * a.Hk + h) * a.S * a.G;
  float *const po = parts.o + (prow + r) * a.Dh;
  T *const y = (T *)a.y + ((long long)b * a.S + qi) * a.ldy + (long long)hq * a.Dh;
  if (plan.parts == 1 && me.l == 0.f) qhi = qlo;  // a row without any weight: zeros, whatever it sees
  if (live) {
    if (plan.parts > 1)
      me.put_part(po, parts.ml + prow + r, a.Dh);
    else
      me.put(y, a.Dh);
  }
  if (!PAGED) return;
  // Values that are no numbers where some rows see them and others not: for the rows that do, into sums of their own, as the
  // kernel's would have to stay in registers for it (4 x 300 positions of 16 heads of 192 behind 2000 172 -> 192 us).  One NaN in 2 x
  // 2048 positions over 8192, 32 heads of 128: 521 -> 557 us.
  __syncthreads();
  if (!dirty) return;
  me.clear();
  for (int t = 0; t < nt; ++t) {
    const int k0 = lo + t * KT;
    if (!mixed(k0)) continue;
    mv.put_again(k0, lds);
    __syncthreads();
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) me.odd_values(lds + TB, kb * 32, k0 + kb * 32 + 4 * (lane >> 5) - qlo, max(qhi - qlo, 0));
    __syncthreads();
  }
  if (!live) return;
  if (plan.parts > 1)
    me.add(po, a.Dh);
  else
    me.add(y, a.Dh);
}

template <typename T, bool PAGED>
hipError_t launch_tiles_as(const MhaArgs &a, TilePlan plan, hipStream_t st) {
  const long long all = (long long)a.B * a.Hk * plan.tiles * plan.parts, most = 1 << 22;  // workgroups of a launch
  for (long long first = 0; first < all; first += most) {
    plan.first = (int)first;
    const dim3 grid((unsigned)(all - first < most ? all - first : most)), block(256);
    if (a.Dh <= 64)
      hipLaunchKernelGGL((tile_kernel<T, 64, PAGED>), grid, block, 0, st, a, plan);
    else if (a.Dh <= 128)
      hipLaunchKernelGGL((tile_kernel<T, 128, PAGED>), grid, block, 0, st, a, plan);
    else
      hipLaunchKernelGGL((tile_kernel<T, 256, PAGED>), grid, block, 0, st, a, plan);
  }
  return hipGetLastError();
}

hipError_t launch_tiles_bf16(const MhaArgs &a, const TilePlan &plan, hipStream_t st);
hipError_t launch_tiles_f32(const MhaArgs &a, const TilePlan &plan, hipStream_t st);

}  // namespace mt
