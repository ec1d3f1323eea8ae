// What mixes the rows of a sequence: host side of lirpa_conv_* and lirpa_scan_*.  Kernels:
// conv.hpp, scan.hpp.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "conv.hpp"
#include "lirpa.h"
#include "lm_host.hpp"
#include "scan.hpp"

using namespace lirpa_host;
using namespace lm;

namespace {

int check_seq(const char* who, const int32_t* seq, int slots) {
  if ((uintptr_t)seq % 4) return fail(LIRPA_EINVAL, "%s: seq is not aligned to its type", who);
  if (slots < 1) return fail(LIRPA_EINVAL, "%s: slots = %d is below 1", who, slots);
  return LIRPA_OK;
}

int too_large(const char* who) {
  return fail(LIRPA_EUNSUPPORTED, "%s: a launch would pass 2^32 threads", who);
}

// ---------------------------------------------------------------------------------------------
// Convolution
// ---------------------------------------------------------------------------------------------
constexpr int kMaxTaps = 8;

template <typename F>
int by_taps(int taps, F&& f) {
  using std::integral_constant;
  switch (taps) {
    case 1: return f(integral_constant<int, 1>{});
    case 2: return f(integral_constant<int, 2>{});
    case 3: return f(integral_constant<int, 3>{});
    case 4: return f(integral_constant<int, 4>{});
    case 5: return f(integral_constant<int, 5>{});
    case 6: return f(integral_constant<int, 6>{});
    case 7: return f(integral_constant<int, 7>{});
    default: return f(integral_constant<int, 8>{});
  }
}

int64_t pieces(int n, int wide) { return (n + wide - 1) / wide; }

// Rows of a strip, at least `least`: with those in front of it and, in the gradient, behind it
// (`more`) a multiple of what is on its way at a time; the fewest of some sizes that leave no more
// than kConvThreads threads.  Forward, 8192 x 4096 bf16: 34 us with 2^18, 44 with 2^17 (strips of
// 32), 37 with 2^19 (of 8); 4099 x 1001 f16: strips of 5 14 us, of 8 16.
constexpr int64_t kConvThreads = (int64_t)1 << 18;
constexpr int kConvLeast = 4, kConvBackLeast = 8;  // a strip of the gradient writes a part of dw
constexpr int kConvMost = 8;                       // times what is on its way: the longest strip
int conv_strip(int64_t rows, int n, int wide, int ahead, int more, int least) {
  int strip = 0;
  for (int m : {2, 3, 4, 5, 6, kConvMost}) {
    strip = m * ahead - more;
    if (strip >= least && (rows + strip - 1) / strip * pieces(n, wide) <= kConvThreads) break;
  }
  return strip;
}

// For any type and up to `rows` rows: it does not fall as rows grow.  There are as many strips as the
// least rows a strip or the threads allow, those of the fewest pieces a row, or what the longest
// strips leave.
size_t conv_bytes(int64_t rows, int n, int taps) {
  const int longest = kConvMost * kConvAhead - 2 * (taps - 1);
  const int64_t allowed = std::min((rows + kConvBackLeast - 1) / kConvBackLeast,
                                   kConvThreads / pieces(n, kConvBackWide<bf16>));
  const int64_t strips = std::max(allowed, (rows + longest - 1) / longest);
  return std::max<size_t>(256, (size_t)strips * (taps + 1) * n * sizeof(float));
}

int check_conv(const char* who, int dtype, int64_t rows, int n, int taps, const void* w,
               const void* bias, int act) {
  TRY(check_shape(who, dtype, rows, n));
  if (taps < 1 || taps > kMaxTaps)
    return fail(LIRPA_EINVAL, "%s: taps = %d is outside [1, %d]", who, taps, kMaxTaps);
  if (act != LIRPA_CONV_LINEAR && act != LIRPA_CONV_SILU)
    return fail(LIRPA_EINVAL, "%s: act %d is none of lirpa_conv_act", who, act);
  if (rows == 0) return LIRPA_OK;
  TRY(check_rows(who, "w", dtype, w, n, n));
  if (bias) TRY(check_rows(who, "bias", dtype, bias, n, n));
  return LIRPA_OK;
}

int check_conv_state(const char* who, int dtype, int n, const void* state, const void* state_out) {
  if (state) TRY(check_rows(who, "state", dtype, state, n, n));
  if (state_out) TRY(check_rows(who, "state_out", dtype, state_out, n, n));
  return LIRPA_OK;
}

template <typename T>
Conv<T> conv_args(int64_t rows, int n, const void* x, int64_t ldx, const void* w, const void* bias,
                  int act, const int32_t* seq, int slots) {
  Conv<T> a{};
  a.x = (const T*)x;
  a.ldx = ldx;
  a.w = (const T*)w;
  a.bias = (const T*)bias;
  a.s = Sequences{seq, rows, slots};
  a.n = n;
  a.silu = act == LIRPA_CONV_SILU;
  return a;
}

// ---------------------------------------------------------------------------------------------
// Scan
// ---------------------------------------------------------------------------------------------
constexpr int kMaxStates = 64;

// Lanes that share a column, four states each.  With eight, half the lanes and twice the chunks the
// real walk of 8192 x 4096 with 16 states gains 7 us of 174, the first one and the link lose 23.
int scan_lanes(int states) { return states <= 8 ? 2 : states <= 16 ? 4 : states <= 32 ? 8 : 16; }

template <typename F>
int by_lanes(int states, F&& f) {
  using std::integral_constant;
  switch (scan_lanes(states)) {
    case 2: return f(integral_constant<int, 2>{});
    case 4: return f(integral_constant<int, 4>{});
    case 8: return f(integral_constant<int, 8>{});
    default: return f(integral_constant<int, 16>{});
  }
}

int64_t scan_groups(int n, int states) {
  const int columns = 256 / scan_lanes(states);
  return (n + columns - 1) / columns;
}

// Rows are cut into chunks until there are kScanBlocks blocks, or kMostChunks chunks: their states
// are linked one after the other.  16 states, bf16, first walk, link and real walk, us (between
// events, which add some 2 to each): 8192 x 4096 129 + 7 + 243 with 512 blocks, 114 + 8 + 185 with
// 1024, 106 + 11 + 181 with 2048; 512 x 1024 with chunks of 16 rows 8 + 9 + 11, of 64 11 + 6 + 18, of
// 256 28 + 6 + 50; 8192 x 256 with 64 chunks 17 + 15 + 29, with 512 14 + 93 + 21.
constexpr int kScanBlocks = 2048, kMostChunks = 64;
int64_t scan_most_chunks(int n, int states) {
  const int64_t groups = scan_groups(n, states);
  return std::clamp<int64_t>((kScanBlocks + groups - 1) / groups, 1, kMostChunks);
}
int64_t scan_chunk(int64_t rows, int n, int states) {
  const int64_t want = scan_most_chunks(n, states);
  return std::max<int64_t>(kSpan, up((rows + want - 1) / want, kSpan));
}

struct ScanRoom {
  float *local, *begin, *deltas, *dA, *dD, *dbias, *dBC;
  int* links;
  size_t bytes;
};
// For the most chunks that up to `rows` rows can be cut into.
ScanRoom scan_room(int64_t rows, int n, int states, bool backward, void* base) {
  Carver ws{(char*)base};
  ScanRoom r{};
  const int padded = 4 * scan_lanes(states);
  const int64_t chunks =
      std::min((rows + kSpan - 1) / kSpan, scan_most_chunks(n, states));
  const size_t column = (size_t)chunks * n * sizeof(float);
  if (chunks > 1) {
    r.local = (float*)ws.take(column * padded);
    if (!backward) r.begin = (float*)ws.take(column * padded);
    r.deltas = (float*)ws.take(column);
    r.links = (int*)ws.take((size_t)chunks * sizeof(int));
  }
  if (backward) {
    r.dA = (float*)ws.take(column * padded);
    r.dD = (float*)ws.take(column);
    r.dbias = (float*)ws.take(column);
    r.dBC = (float*)ws.take((size_t)scan_groups(n, states) * rows * 2 * padded * sizeof(float));
  }
  r.bytes = std::max<size_t>(256, ws.at);
  return r;
}

int check_scan(const char* who, const lirpa_scan* s) {
  if (!s) return fail(LIRPA_EINVAL, "%s: the scan is null", who);
  TRY(check_shape(who, s->dtype, s->rows, s->n));
  if (s->states < 1 || s->states > kMaxStates)
    return fail(LIRPA_EINVAL, "%s: states = %d is outside [1, %d]", who, s->states, kMaxStates);
  if (s->rows == 0) return LIRPA_OK;
  TRY(check_rows(who, "u", s->dtype, s->u, s->ldu, s->n));
  TRY(check_rows(who, "dt", s->dtype, s->dt, s->lddt, s->n));
  if (s->z) TRY(check_rows(who, "z", s->dtype, s->z, s->ldz, s->n));
  TRY(check_rows(who, "B", s->dtype, s->B, s->ldB, s->states));
  TRY(check_rows(who, "C", s->dtype, s->C, s->ldC, s->states));
  TRY(check_floats(who, "A", s->A, true));
  TRY(check_floats(who, "D", s->D, false));
  TRY(check_floats(who, "bias", s->bias, false));
  return check_seq(who, s->seq, s->slots);
}

template <typename T>
Scan<T> scan_args(const lirpa_scan* s) {
  Scan<T> a{};
  a.u = (const T*)s->u;
  a.dt = (const T*)s->dt;
  a.z = (const T*)s->z;
  a.B = (const T*)s->B;
  a.C = (const T*)s->C;
  a.A = s->A;
  a.D = s->D;
  a.bias = s->bias;
  a.ldu = s->ldu;
  a.lddt = s->lddt;
  a.ldz = s->ldz;
  a.ldB = s->ldB;
  a.ldC = s->ldC;
  a.s = Sequences{s->seq, s->rows, s->slots};
  a.n = s->n;
  a.states = s->states;
  return a;
}

template <typename T>
void use_room(Scan<T>& a, const ScanRoom& r) {
  a.local = r.local;
  a.begin = r.begin;
  a.deltas = r.deltas;
  a.links = r.links;
  a.dA = r.dA;
  a.dD = r.dD;
  a.dbias = r.dbias;
  a.dBC = r.dBC;
  a.chunk = (int)scan_chunk(a.s.rows, a.n, a.states);
  a.chunks = (int)((a.s.rows + a.chunk - 1) / a.chunk);
}

template <typename T, int LANES>
int scan_forward(Scan<T> a, hipStream_t st) {
  const int groups = (int)scan_groups(a.n, a.states);
  const int64_t blocks = (int64_t)groups * a.chunks;
  if (blocks > max_blocks(256)) return too_large("lirpa_scan_forward");
  if (a.chunks > 1) {
    TRY(launch_k("scan_local", st, [&] {
      k_scan_local<T, LANES><<<(unsigned)(blocks - groups), 256, 0, st>>>(a, groups);
    }));
    TRY(launch_k("scan_link", st, [&] {
      k_scan_link<T, LANES, false><<<(a.n * LANES + 255) / 256, 256, 0, st>>>(a);
    }));
  }
  return launch_k("scan_forward", st, [&] {
    k_scan_fwd<T, LANES><<<(unsigned)blocks, 256, 0, st>>>(a, groups);
  });
}

template <typename T, int LANES>
int scan_backward(Scan<T> a, T* dB, int64_t lddB, T* dC, int64_t lddC, float* dA, float* dD,
                  float* dbias, hipStream_t st) {
  const int groups = (int)scan_groups(a.n, a.states), padded = 4 * LANES;
  const int64_t blocks = (int64_t)groups * a.chunks;
  const int64_t vectors = (a.s.rows * 2 * padded + 255) / 256;
  if (std::max(blocks, vectors) > max_blocks(256)) return too_large("lirpa_scan_backward");
  if (a.chunks > 1) {
    TRY(launch_k("scan_back_local", st, [&] {
      k_scan_back_local<T, LANES><<<(unsigned)(blocks - groups), 256, 0, st>>>(a, groups);
    }));
    TRY(launch_k("scan_link", st, [&] {
      k_scan_link<T, LANES, true><<<(a.n * LANES + 255) / 256, 256, 0, st>>>(a);
    }));
  }
  TRY(launch_k("scan_backward", st, [&] {
    k_scan_bwd<T, LANES><<<(unsigned)blocks, 256, 0, st>>>(a, groups);
  }));
  TRY(launch_k("scan_vectors", st, [&] {
    k_scan_vectors<T><<<(unsigned)vectors, 256, 0, st>>>(a.dBC, groups, a.s.rows, padded, a.states,
                                                         dB, lddB, dC, lddC);
  }));
  if (!dA && !dD && !dbias) return LIRPA_OK;
  return launch_k("scan_sums", st, [&] {
    const int64_t values = (int64_t)a.n * (padded + 2);
    k_scan_sums<<<(unsigned)((values + 255) / 256), 256, 0, st>>>(
        a.dA, a.dD, a.dbias, a.chunks, a.n, padded, a.states, dA, dD, dbias);
  });
}

}  // namespace

extern "C" {

int lirpa_conv_forward(int dtype, int64_t rows, int n, int taps, const void* x, int64_t ldx,
                       const void* w, const void* bias, int act, const int32_t* seq, int slots,
                       const void* state, void* state_out, void* y, int64_t ldy,
                       hipStream_t stream) {
  return guarded([&] {
    const char* who = "lirpa_conv_forward";
    TRY(check_conv(who, dtype, rows, n, taps, w, bias, act));
    TRY(check_seq(who, seq, slots));
    if (rows == 0) return (int)LIRPA_OK;
    TRY(check_rows(who, "x", dtype, x, ldx, n));
    TRY(check_rows(who, "y", dtype, y, ldy, n));
    TRY(check_conv_state(who, dtype, n, state, state_out));
    return by_type(dtype, [&](auto t) {
      using T = decltype(t);
      Conv<T> a = conv_args<T>(rows, n, x, ldx, w, bias, act, seq, slots);
      a.state = (const T*)state;
      a.state_out = (T*)state_out;
      a.y = (T*)y;
      a.ldy = ldy;
      constexpr int wide = kConvWide<T>;
      a.strip = conv_strip(rows, n, wide, kConvAhead, taps - 1, kConvLeast);
      const int64_t strips = (rows + a.strip - 1) / a.strip;
      const int64_t blocks = (strips * pieces(n, wide) + 255) / 256;
      const int64_t slabs = (pieces(n, wide) + 255) / 256, ends = (rows + 63) / 64 * slabs;
      if (std::max(blocks, ends) > max_blocks(256)) return too_large(who);
      return by_taps(taps, [&](auto k) {
        TRY(launch_k("conv_forward", stream, [&] {
          k_conv_fwd<T, k.value><<<(unsigned)blocks, 256, 0, stream>>>(a);
        }));
        if (!state_out || taps == 1) return (int)LIRPA_OK;
        return launch_k("conv_state", stream, [&] {
          k_conv_state<T, k.value><<<(unsigned)ends, 256, 0, stream>>>(a, (int)slabs);
        });
      });
    });
  });
}

int lirpa_conv_step(int dtype, int64_t rows, int n, int taps, const void* x, int64_t ldx,
                    const void* w, const void* bias, int act, const int32_t* seq, int slots,
                    const void* state, void* state_out, void* y, int64_t ldy, hipStream_t stream) {
  return guarded([&] {
    const char* who = "lirpa_conv_step";
    TRY(check_conv(who, dtype, rows, n, taps, w, bias, act));
    TRY(check_seq(who, seq, slots));
    if (rows == 0) return (int)LIRPA_OK;
    TRY(check_rows(who, "x", dtype, x, ldx, n));
    TRY(check_rows(who, "y", dtype, y, ldy, n));
    TRY(check_conv_state(who, dtype, n, state, state_out));
    return by_type(dtype, [&](auto t) {
      using T = decltype(t);
      Conv<T> a = conv_args<T>(rows, n, x, ldx, w, bias, act, seq, slots);
      a.state = (const T*)state;
      a.state_out = (T*)state_out;
      a.y = (T*)y;
      a.ldy = ldy;
      const int64_t blocks = (rows * pieces(n, kConvWide<T>) + 255) / 256;
      if (blocks > max_blocks(256)) return too_large(who);
      return by_taps(taps, [&](auto k) {
        return launch_k("conv_step", stream, [&] {
          k_conv_step<T, k.value><<<(unsigned)blocks, 256, 0, stream>>>(a);
        });
      });
    });
  });
}

size_t lirpa_conv_workspace_bytes(int64_t rows, int n, int taps) {
  if (rows < 0 || rows > kMaxRows || n < 1 || n > kMaxWidth || taps < 1 || taps > kMaxTaps)
    return 0;
  return conv_bytes(rows, n, taps);
}

int lirpa_conv_backward(int dtype, int64_t rows, int n, int taps, const void* dy, int64_t lddy,
                        const void* x, int64_t ldx, const void* w, const void* bias, int act,
                        const int32_t* seq, int slots, void* dx, int64_t lddx, void* dw,
                        void* dbias, void* ws, size_t ws_bytes, hipStream_t stream) {
  return guarded([&] {
    const char* who = "lirpa_conv_backward";
    TRY(check_conv(who, dtype, rows, n, taps, w, bias, act));
    TRY(check_seq(who, seq, slots));
    if (rows > 0) {
      TRY(check_rows(who, "dy", dtype, dy, lddy, n));
      TRY(check_rows(who, "x", dtype, x, ldx, n));
      TRY(check_rows(who, "dx", dtype, dx, lddx, n));
    }
    TRY(check_rows(who, "dw", dtype, dw, n, n));
    if (dbias) TRY(check_rows(who, "dbias", dtype, dbias, n, n));
    TRY(check_ws(who, ws, ws_bytes, lirpa_conv_workspace_bytes(rows, n, taps)));
    return by_type(dtype, [&](auto t) {
      using T = decltype(t);
      Conv<T> a = conv_args<T>(rows, n, x, ldx, w, bias, act, seq, slots);
      a.dy = (const T*)dy;
      a.lddy = lddy;
      a.dx = (T*)dx;
      a.lddx = lddx;
      constexpr int wide = kConvBackWide<T>;
      a.strip = conv_strip(rows, n, wide, kConvAhead, 2 * (taps - 1),
                           kConvBackLeast);
      a.part = (float*)ws;
      const int64_t strips = (rows + a.strip - 1) / a.strip, ld = (int64_t)(taps + 1) * n;
      const int64_t blocks = (strips * pieces(n, wide) + 255) / 256;
      if (blocks > max_blocks(256)) return too_large(who);
      if (rows > 0)
        TRY(by_taps(taps, [&](auto k) {
          return launch_k("conv_backward", stream, [&] {
            k_conv_bwd<T, k.value><<<(unsigned)blocks, 256, 0, stream>>>(a);
          });
        }));
      return launch_k("conv_dw", stream, [&] {
        const int64_t values = dbias ? ld : (int64_t)taps * n;
        k_sum_parts<T><<<(unsigned)((values + 31) / 32), 256, 0, stream>>>(
            a.part, strips, ld, values, (int64_t)taps * n, (T*)dw, (T*)dbias);
      });
    });
  });
}

size_t lirpa_scan_workspace_bytes(int64_t rows, int n, int states, int backward) {
  if (rows < 0 || rows > kMaxRows || n < 1 || n > kMaxWidth || states < 1 ||
      states > kMaxStates || (backward != 0 && backward != 1))
    return 0;
  return scan_room(rows, n, states, backward == 1, nullptr).bytes;
}

size_t lirpa_scan_kept_bytes(int64_t rows, int n, int states) {
  if (rows < 0 || rows > kMaxRows || n < 1 || n > kMaxWidth || states < 1 || states > kMaxStates)
    return 0;
  return std::max<size_t>(
      16, (size_t)((rows + kSpan - 1) / kSpan) * n * 4 * scan_lanes(states) * sizeof(float));
}

int lirpa_scan_forward(const lirpa_scan* scan, const float* state, float* state_out, void* y,
                       int64_t ldy, void* kept, void* ws, size_t ws_bytes, hipStream_t stream) {
  return guarded([&] {
    const char* who = "lirpa_scan_forward";
    TRY(check_scan(who, scan));
    if (scan->rows == 0) return (int)LIRPA_OK;
    TRY(check_floats(who, "state", state, false));
    TRY(check_floats(who, "state_out", state_out, false));
    TRY(check_rows(who, "y", scan->dtype, y, ldy, scan->n));
    if (kept && state)
      return fail(LIRPA_EINVAL, "%s: the backward pass starts from states of 0, not from state",
                  who);
    if (!aligned16(kept))
      return fail(LIRPA_EINVAL, "%s: kept does not start on 16 bytes", who);
    TRY(check_ws(who, ws, ws_bytes,
                 lirpa_scan_workspace_bytes(scan->rows, scan->n, scan->states, 0)));
    return by_type(scan->dtype, [&](auto t) {
      using T = decltype(t);
      Scan<T> a = scan_args<T>(scan);
      use_room(a, scan_room(scan->rows, scan->n, scan->states, false, ws));
      a.state = state;
      a.state_out = state_out;
      a.y = (T*)y;
      a.ldy = ldy;
      a.kept = (float*)kept;
      return by_lanes(scan->states,
                      [&](auto lanes) { return scan_forward<T, lanes.value>(a, stream); });
    });
  });
}

int lirpa_scan_step(const lirpa_scan* scan, const float* state, float* state_out, void* y,
                    int64_t ldy, hipStream_t stream) {
  return guarded([&] {
    const char* who = "lirpa_scan_step";
    TRY(check_scan(who, scan));
    if (scan->rows == 0) return (int)LIRPA_OK;
    TRY(check_floats(who, "state", state, false));
    TRY(check_floats(who, "state_out", state_out, false));
    TRY(check_rows(who, "y", scan->dtype, y, ldy, scan->n));
    return by_type(scan->dtype, [&](auto t) {
      using T = decltype(t);
      Scan<T> a = scan_args<T>(scan);
      a.state = state;
      a.state_out = state_out;
      a.y = (T*)y;
      a.ldy = ldy;
      const int64_t groups = scan_groups(a.n, a.states), blocks = groups * scan->rows;
      if (blocks > max_blocks(256)) return too_large(who);
      return by_lanes(scan->states, [&](auto lanes) {
        return launch_k("scan_step", stream, [&] {
          k_scan_step<T, lanes.value><<<(unsigned)blocks, 256, 0, stream>>>(a, (int)groups);
        });
      });
    });
  });
}

int lirpa_scan_backward(const lirpa_scan* scan, const void* dy, int64_t lddy, const void* kept,
                        void* du, int64_t lddu, void* ddt, int64_t ldddt, void* dz, int64_t lddz,
                        void* dB, int64_t lddB, void* dC, int64_t lddC, float* dA, float* dD,
                        float* dbias, void* ws, size_t ws_bytes, hipStream_t stream) {
  return guarded([&] {
    const char* who = "lirpa_scan_backward";
    TRY(check_scan(who, scan));
    const int64_t rows = scan->rows;
    const int dtype = scan->dtype, n = scan->n, states = scan->states;
    if (rows > 0) {
      TRY(check_rows(who, "dy", dtype, dy, lddy, n));
      if (!kept) return fail(LIRPA_EINVAL, "%s: kept is null", who);
      if (!aligned16(kept)) return fail(LIRPA_EINVAL, "%s: kept does not start on 16 bytes", who);
      TRY(check_rows(who, "du", dtype, du, lddu, n));
      TRY(check_rows(who, "ddt", dtype, ddt, ldddt, n));
      if (!scan->z != !dz) return fail(LIRPA_EINVAL, "%s: dz goes with z", who);
      if (dz) TRY(check_rows(who, "dz", dtype, dz, lddz, n));
      TRY(check_rows(who, "dB", dtype, dB, lddB, states));
      TRY(check_rows(who, "dC", dtype, dC, lddC, states));
    }
    TRY(check_floats(who, "dA", dA, false));
    TRY(check_floats(who, "dD", dD, false));
    TRY(check_floats(who, "dbias", dbias, false));
    TRY(check_ws(who, ws, ws_bytes, lirpa_scan_workspace_bytes(rows, n, states, 1)));
    if (rows == 0) {  // sums over no rows
      const int padded = 4 * scan_lanes(states);
      if (!dA && !dD && !dbias) return (int)LIRPA_OK;
      return launch_k("scan_sums", stream, [&] {
        const int64_t values = (int64_t)n * (padded + 2);
        k_scan_sums<<<(unsigned)((values + 255) / 256), 256, 0, stream>>>(
            nullptr, nullptr, nullptr, 0, n, padded, states, dA, dD, dbias);
      });
    }
    return by_type(dtype, [&](auto t) {
      using T = decltype(t);
      Scan<T> a = scan_args<T>(scan);
      use_room(a, scan_room(rows, n, states, true, ws));
      a.dy = (const T*)dy;
      a.lddy = lddy;
      a.kept = (float*)kept;
      a.du = (T*)du;
      a.ddt = (T*)ddt;
      a.dz = (T*)dz;
      a.lddu = lddu;
      a.ldddt = ldddt;
      a.lddz = lddz;
      return by_lanes(states, [&](auto lanes) {
        return scan_backward<T, lanes.value>(a, (T*)dB, lddB, (T*)dC, lddC, dA, dD, dbias, stream);
      });
    });
  });
}

}  // extern "C"
