// C ABI of libpotattn (declared in include/pot_attn.h).
//
// Every check runs on the host before any HIP call; a rejected call touches
// neither the device nor the stream. Launches are asynchronous on the
// caller's stream and allocate nothing.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <chrono>
#include <cstdarg>
#include <cstdio>
#include <string>

#include "pot_attn.h"
#include "pot_device.hpp"
#include "pot_launch.hpp"

using namespace potattn;

namespace {

thread_local std::string g_last_error;

pot_status fail(pot_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_last_error = buf;
  return st;
}

}  // namespace

pot_status potattn::report_error(pot_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_last_error = buf;
  return st;
}

namespace {

pot_status ok() {
  g_last_error.clear();
  return POT_OK;
}

pot_status hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return ok();
  return fail(POT_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

constexpr int kE = 6;
constexpr int kMaxF = 12;

pot_status check_format(const pot_format* f) {
  if (!f) return fail(POT_ERR_INVALID_ARG, "fmt is NULL");
  if (f->head_dim != 64) return fail(POT_ERR_UNSUPPORTED, "head_dim %d (only 64)", f->head_dim);
  if (f->exp_bits != 3) return fail(POT_ERR_UNSUPPORTED, "exp_bits %d (only 3)", f->exp_bits);
  if (f->mant_bits < 0 || f->mant_bits > 4)
    return fail(POT_ERR_UNSUPPORTED, "mant_bits %d (0..4)", f->mant_bits);
  if (f->frac_bits < kE)
    return fail(POT_ERR_INVALID_ARG,
                "frac_bits %d < E = %d: a shift F - e would be a right shift", f->frac_bits, kE);
  if (f->frac_bits > kMaxF)
    return fail(POT_ERR_UNSUPPORTED, "frac_bits %d > %d (int32 head-room)", f->frac_bits, kMaxF);
  if (f->hadamard != 0 && f->hadamard != 1)
    return fail(POT_ERR_INVALID_ARG, "hadamard %d (0 or 1)", f->hadamard);
  return POT_OK;
}

struct Plan {
  int n_splits, split_len;
};

// S key splits of T keys, in whole 256-key tiles.
Plan plan_from_count(int T, int S) {
  const int tiles = (T + kTile - 1) / kTile;
  S = std::max(1, std::min(S, tiles));
  const int tiles_per_split = (tiles + S - 1) / S;
  Plan p;
  p.split_len = tiles_per_split * kTile;
  p.n_splits = (T + p.split_len - 1) / p.split_len;
  return p;
}

int split_count_for_slots(long units, long slots) {
  return units >= slots ? 1 : (int)(slots / units);
}

// Upper bound used to size workspaces without a device query: 256 CUs x 8
// resident workgroups (the decode kernels reach at most 4 per CU: 4 waves per SIMD).
constexpr long kMaxSlots = 256L * 8;

Plan plan_bound(int B, int Hkv, int T) {
  return plan_from_count(T, split_count_for_slots((long)B * Hkv, kMaxSlots));
}

std::atomic<int> g_cus[64];
int device_cus() {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) dev = 0;
  int cus = g_cus[dev].load(std::memory_order_relaxed);
  if (cus <= 0) {
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess ||
        cus <= 0)
      cus = 256;
    g_cus[dev].store(cus, std::memory_order_relaxed);
  }
  return cus;
}

// How a decode call is split: (batch, kv head) units times key splits, on
// four-wave or CU-wide (pw waves, 0: the engine has none) workgroups. Figures:
// graph replays, us, eight heads to a unit, PoT-4 over fp16 values unless said.
//  - Up to one unit per CU: CU-wide workgroups and as many splits as give every
//    CU at most one. More splits cost a second round of prologues, fewer leave
//    CUs idle; four-wave workgroups take longer over the prologue (two heads'
//    queries per wave) and the merge. 64 units T = 4096 11.7 with 4 splits, 14.7
//    with 8 on four waves, 15.3 with 4; 24 units T = 16384 16.1 with 10, 18.4 with
//    32 on four waves; the fp16 comparator (four waves) at 96 units 69.4, 78.0
//    with 4.
//  - That rule rounds down: from half the CUs on it leaves one workgroup per unit
//    and the other CUs without work. For long ranges (from 12288 keys; at 8192 one
//    workgroup is as fast, 132 units 36.7 and 36.5) the fp16 comparator and the
//    engines that are bound by their issue take three splits of four-wave
//    workgroups up to two thirds of the CUs (T = 16384, 160 units: PoT-M1 80.4 ->
//    76.5, PoT-M4 108 -> 93, fp16 119.9 -> 108.4), PoT-4 and INT8 keys over fp16 values,
//    whose stream decides sooner, up to three fifths (132 units 68.6 -> 63.4, 152
//    72.2 -> 70.3, 168 75.2 and 77.8). With INT8 values, where a unit takes a CU the
//    longest, three to four workgroups per CU up to three quarters (132 units 68.0
//    -> 55.1, 160 69.8 -> 61.2, 176 70.7 -> 66.9, 192 72.8 -> 67.7; T = 8192 38.0 ->
//    32.5 and 39.6 -> 40.7), and with 4-bit values the same (132 units 46.1 -> 39.2, 160
//    46.5 -> 42.7, 176 48.3 -> 46.3, 192 49.1 -> 47.9; the best counts 38.1, 42.6, 46.3, 47.5).
//  - Where every wave of one workgroup has at most one 64-key tile, one split
//    and no merge: up to 768 keys (T = 512, 4 units 5.8 against 6.8 with two
//    splits, 64 units 6.1 against 7.2; T = 768, 4 units 6.6 against 6.9 with three;
//    on 12 waves PoT-M4 7.4 and 7.6 at 512, but 8.9 and 7.9 at 768), and up to 16
//    tiles on 16 waves if a quarter of the CUs has a unit (T = 1024: 16 units 7.6
//    against 7.2 with four splits, 64 units 7.8 and 7.8, 128 units 8.0 against 9.0
//    with two).
//  - More units than CUs: one split of four-wave workgroups, several of which
//    share a CU, for up to 8191 keys (512 units: T = 256 8.1 against 10.3 CU-wide,
//    T = 4096 57.4 against 59.9; 320 units 41.8 against 47.1); CU-wide above, whose
//    waves claim tiles (512 units, T = 16384 205 against 208), in three splits where
//    those make at most four rounds instead of two whole ones (T = 16384, 320 units
//    145 against 159 with one; 352 units, a fifth round, 168 against 162).
//  - A length per sequence (4-bit values), up to one unit per CU: four four-wave workgroups
//    for every CU, from 1000 keys a split and, where one CU-wide workgroup a unit leaves less
//    than a quarter of the CUs idle, from 1500. They belong to several sequences (four of them
//    are on a CU at once, three at k = 3 and 4), so that what a short one leaves serves the
//    others. The lengths are not known here: ones that differ gain, equal ones lose where the
//    other plan leaves no CU idle. us, here / by the rules above, for lengths from T down to
//    T/B in equal steps, all T, every other one T/8, all but one T/8:
//      64 units T = 16384 PoT-4   17.5/19.6  22.9/21.1  21.8/19.3  14.6/18.2
//      64 units T = 16384 PoT-M4  25.6/28.0  34.0/29.8  30.4/28.5  18.5/26.8
//      96 units T = 10240 PoT-4   17.1/21.2  22.7/22.2  20.1/21.0  14.6/20.1
//      160 units T = 6144 PoT-4   17.7/21.5  23.1/22.4  20.8/21.7  14.9/20.3
//      160 units T = 6144 PoT-M4  26.8/34.9  34.0/35.7  33.0/35.1  17.6/33.8
//      256 units T = 8192 PoT-4   26.3/27.7  37.4/30.9  34.4/27.8  21.0/24.6
//    and with fewer keys a split than that:
//      64 units T = 8192 PoT-4    14.4/13.7  16.8/14.9  16.1/13.7  12.4/12.8
//      256 units T = 5120 PoT-4   21.5/19.6  27.8/21.6  25.6/20.4  16.7/18.1
//      256 units T = 4096 PoT-4   19.0/17.7  24.4/19.3  23.0/17.8  15.6/16.4
//    More units than CUs: 400 units T = 16384 59.4/50.2 in equal steps.
constexpr int kShortKeys = 768, kLongKeys = 8192, kSpreadKeys = 12288;
constexpr int kRaggedKeys = 1000, kRaggedKeysFull = 1500;
struct Launch {
  Plan plan;
  bool pool;
};

// Splits of four-wave workgroups, over two and up to four to a CU, that leave the
// smallest share of the CUs' places empty.
int spread_splits(long units, long cus) {
  int best = 1;
  long best_used = 0, best_places = 1;
  for (long S = 2 * cus / units + 1; S * units <= 4 * cus; ++S) {
    const long used = S * units, places = (used + cus - 1) / cus * cus;
    if (used * best_places > best_used * places) {
      best = (int)S;
      best_used = used;
      best_places = places;
    }
  }
  return best;
}

// What of an engine the plan depends on.
struct PlanEngine {
  int pw;            // waves of its CU-wide workgroups, 0: none
  bool int8_values;  // or 4-bit ones
  bool light;        // PoT-4 or INT8 keys over fp16 values: the stream decides even on one CU
  bool ragged;       // a length per sequence
};

Launch plan_launch(long units, int T, const PlanEngine& e, int cus, int bound) {
  const int pw = e.pw;
  const bool one_tile = pw > 0 && (T <= kShortKeys || (T <= pw * 64 && 4 * units >= cus));
  int S = 1;
  bool pool = pw > 0;
  if (e.ragged && units <= cus) {
    const long S4 = 4L * cus / units;
    if (T >= (4 * units > 3L * cus ? kRaggedKeysFull : kRaggedKeys) * S4) return {plan_from_count(T, (int)std::min(S4, (long)bound)), false};
  }
  if (units <= cus) {
    if (!one_tile) S = (int)(cus / units);
    if (S == 1 && T >= kSpreadKeys) {
      if (e.int8_values ? 4 * units <= 3L * cus
                        : (e.light ? 5 * units <= 3L * cus : 3 * units <= 2L * cus)) {
        S = e.int8_values ? spread_splits(units, cus) : 3;
        pool = false;
      }
    }
  } else {
    pool = pool && T >= kLongKeys;
    if (pool && 3 * units <= 4L * cus) S = 3;
  }
  return {plan_from_count(T, std::min(S, bound)), pool};
}

// CU-wide workgroups claim their tiles from a counter when the grid fills the
// chip and every wave has over four (long streams drift apart, graph replays of 256
// units at T = 32768: PoT-4 203 us against 209 in fixed order, PoT-M4 247 against
// 259, PoT-4 over INT8 values 145 against 163; four tiles per wave, 64 units at T =
// 16384: 33.2 against 32.9). In fixed order the sums are the same from call to call.
bool claims_tiles(long units, const Plan& p, int pw, int cus) {
  return units * p.n_splits >= cus && p.split_len > 4 * pw * 64;
}

size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

struct WsLayout {
  size_t part_m, part_l, part_o, total;
};

// Workspace: query_words per decode workgroup (the tickets are in them), then the
// split partials.
WsLayout ws_layout(long B, long Hq, long Hkv, long S) {
  WsLayout w;
  w.part_m = align_up((size_t)(B * Hkv * S) * query_words((int)(Hq / Hkv)) * 4, 256);
  w.part_l = w.part_m + align_up((size_t)(B * Hq * S) * 4, 256);
  w.part_o = w.part_l + align_up((size_t)(B * Hq * S) * 4, 256);
  w.total = w.part_o + align_up((size_t)(B * Hq * S) * 64 * 4, 256);
  return w;
}

// A tag that a workspace does not hold by chance: 52 bits, never 0, another one
// for each call.
unsigned long long next_ticket() {
  static std::atomic<unsigned long long> n{
      (unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count()};
  unsigned long long z = n.fetch_add(0x9E3779B97F4A7C15ull, std::memory_order_relaxed);
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;  // splitmix64
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  z = (z ^ (z >> 31)) >> 12;
  return z != 0 ? z : 1;
}

bool shape_ok(int B, int Hq, int Hkv, int T) {
  return B >= 1 && Hq >= 1 && Hkv >= 1 && T >= 1 && Hq % Hkv == 0;
}

// Validates the GQA head map and fills DecodeArgs::q_of_kv ([Hkv][G]).
pot_status check_heads(const int32_t* map, int Hq, int Hkv, DecodeArgs* a, int* G_out) {
  if (!map) return fail(POT_ERR_INVALID_ARG, "kv_head_of_q is NULL");
  if (Hq > kMaxHqArg) return fail(POT_ERR_UNSUPPORTED, "Hq %d > %d", Hq, kMaxHqArg);
  if (Hq % Hkv) return fail(POT_ERR_UNSUPPORTED, "Hq %d not a multiple of Hkv %d", Hq, Hkv);
  const int G = Hq / Hkv;
  if (G != 1 && G != 2 && G != 4 && G != 8)
    return fail(POT_ERR_UNSUPPORTED, "group size %d (1, 2, 4 or 8)", G);
  int fill[kMaxHqArg] = {};
  for (int i = 0; i < Hq; ++i) {
    const int h = map[i];
    if (h < 0 || h >= Hkv)
      return fail(POT_ERR_INVALID_ARG, "kv_head_of_q[%d] = %d outside [0, %d)", i, h, Hkv);
    if (fill[h] >= G)
      return fail(POT_ERR_UNSUPPORTED, "kv head %d serves more than %d query heads", h, G);
    const int at = h * G + fill[h]++;
    a->q_of_kv[at >> 2] |= (uint32_t)i << (8 * (at & 3));
  }
  *G_out = G;
  return POT_OK;
}

// Shared tail of the three decode entry points.
pot_status decode_common(int mode, int mant_bits, DecodeArgs& a, const int32_t* map, int B,
                         int Hq, int Hkv, int T, int64_t t_cap, void* workspace,
                         size_t ws_bytes, pot_debug* dbg, void* stream, int vf = 0) {
  const bool v8 = vf != 0;
  if (!shape_ok(B, Hq, Hkv, T))
    return fail(POT_ERR_INVALID_ARG, "bad shape B=%d Hq=%d Hkv=%d T=%d", B, Hq, Hkv, T);
  if (t_cap < T) return fail(POT_ERR_INVALID_ARG, "T %d > t_cap %lld", T, (long long)t_cap);
  if (T > kMaxKeys)
    return fail(POT_ERR_UNSUPPORTED, "T %d > %d keys per sequence (32-bit buffer ranges)", T,
                kMaxKeys);
  if (t_cap % 8)
    return fail(POT_ERR_INVALID_ARG, "t_cap %lld is not a multiple of 8 (value-cache groups)",
                (long long)t_cap);
  if (vf == 3) {
    if (!a.q || !a.v4 || !a.out) return fail(POT_ERR_INVALID_ARG, "q, v_u4 or out is NULL");
    if (!aligned(a.q, 16) || !aligned(a.v4, 16) || !aligned(a.out, 16))
      return fail(POT_ERR_INVALID_ARG, "q, v_u4 and out must be 16-byte aligned");
    if (!aligned(a.seq_lens, 4))
      return fail(POT_ERR_INVALID_ARG, "seq_lens must be 4-byte aligned");
  } else if (v8) {
    if (!a.q || !a.v8 || !a.v_exp || !a.out)
      return fail(POT_ERR_INVALID_ARG, "q, v_u8, v_exp or out is NULL");
    if (!aligned(a.q, 16) || !aligned(a.v8, 16) || !aligned(a.v_exp, 16) || !aligned(a.out, 16))
      return fail(POT_ERR_INVALID_ARG, "q, v_u8, v_exp and out must be 16-byte aligned");
  } else {
    if (!a.q || !a.v || !a.out) return fail(POT_ERR_INVALID_ARG, "q, v or out is NULL");
    if (!aligned(a.q, 16) || !aligned(a.v, 16) || !aligned(a.out, 16))
      return fail(POT_ERR_INVALID_ARG, "q, v and out must be 16-byte aligned");
  }
  if (!workspace) return fail(POT_ERR_INVALID_ARG, "workspace is NULL");
  if (!aligned(workspace, 256))
    return fail(POT_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  int G = 0;
  pot_status st = check_heads(map, Hq, Hkv, &a, &G);
  if (st != POT_OK) return st;
  const int force = dbg ? dbg->force_splits : 0;
  if (force < 0) return fail(POT_ERR_INVALID_ARG, "force_splits %d < 0", force);
  const int mbits = (mode == kScorePot || mode == kScoreDs4a) ? mant_bits : 0;
  const int pw = pool_waves(mode, mbits, vf);
  const int want = dbg ? dbg->force_wg_waves : 0;
  if (want != 0 && want != kBlock / 64 && (pw == 0 || want != pw))
    return fail(POT_ERR_INVALID_ARG, "force_wg_waves %d is neither 0, %d nor %d", want,
                kBlock / 64, pw);
  const long units = (long)B * Hkv;
  const int cus = device_cus();
  Plan p;
  bool pool;
  if (force > 0) {
    p = plan_from_count(T, force);
    pool = pw > 0 && want != kBlock / 64 && (want == pw || units * p.n_splits <= cus);
  } else {
    const PlanEngine e{want == kBlock / 64 ? 0 : pw, v8,
                       mbits == 0 && mode != kScoreFp16 && !v8, a.seq_lens != nullptr};
    const Launch l = plan_launch(units, T, e, cus, plan_bound(B, Hkv, T).n_splits);
    p = l.plan;
    pool = pw > 0 && (want == pw || l.pool);
  }
  const WsLayout w = ws_layout(B, Hq, Hkv, p.n_splits);
  if (ws_bytes < w.total)
    return fail(POT_ERR_WORKSPACE, "workspace %zu bytes < %zu needed for %d splits", ws_bytes,
                w.total, p.n_splits);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  a.tickets = reinterpret_cast<unsigned long long*>(ws);
  a.ticket = pool && p.n_splits > 1 && p.n_splits <= kMaxMergedSplits ? next_ticket() : 0;
  a.part_m = reinterpret_cast<int32_t*>(ws + w.part_m);
  a.part_l = reinterpret_cast<float*>(ws + w.part_l);
  a.part_o = reinterpret_cast<float*>(ws + w.part_o);
  a.t_cap = t_cap;
  a.B = B;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.T = T;
  a.n_splits = p.n_splits;
  a.split_len = p.split_len;
  a.wg_waves = pool ? pw : kBlock / 64;
  a.claim_tiles = pool && claims_tiles(units, p, pw, cus);
  bool debug = false;
  hipEvent_t ev_begin = nullptr, ev_end = nullptr;
  if (dbg) {
    ev_begin = static_cast<hipEvent_t>(dbg->decode_begin);
    ev_end = static_cast<hipEvent_t>(dbg->decode_end);
    a.dbg_qhat = dbg->qhat;
    a.dbg_delta = dbg->delta;
    a.dbg_scores = dbg->scores;
    a.dbg_m_final = dbg->m_final;
    a.dbg_m_split = dbg->m_split;
    debug = dbg->qhat || dbg->delta || dbg->scores || dbg->m_final || dbg->m_split;
    dbg->n_splits = p.n_splits;
    dbg->split_len = p.split_len;
    dbg->wg_waves = a.wg_waves;
    if (debug && mode == kScoreFp16)
      return fail(POT_ERR_UNSUPPORTED, "debug taps are not available on the fp16 path");
    if (debug && vf == 3)
      return fail(POT_ERR_UNSUPPORTED, "debug taps are not available with 4-bit values");
  }
  return hip_status(
      launch_decode(mode, G, mant_bits, debug, vf, a, static_cast<hipStream_t>(stream), ev_begin,
                    ev_end),
      "decode launch");
}

// Shared body of the INT8-value entry points; vf 1: softmax weights, 2:
// power-of-two weights.
pot_status decode_v8(int vf, const pot_format* fmt, int32_t engine, const float* q,
                                   const uint8_t* codes_se, const uint8_t* codes_m,
                                   const float* key_scale, const uint8_t* v_u8,
                                   const int8_t* v_exp, int64_t t_cap,
                                   const int32_t* kv_head_of_q, int32_t B, int32_t Hq,
                                   int32_t Hkv, int32_t T, float* out, void* workspace,
                                   size_t ws_bytes, pot_debug* dbg, void* stream) {
  pot_status st = check_format(fmt);
  if (st != POT_OK) return st;
  if (engine != 0 && engine != 1)
    return fail(POT_ERR_INVALID_ARG, "engine %d (0 shift-accumulate, 1 byte decode)", engine);
  if (engine == 1 && fmt->mant_bits != 0)
    return fail(POT_ERR_UNSUPPORTED, "the byte-decode path scores PoT-4 codes only (mant_bits 0)");
  if (!codes_se || !key_scale) return fail(POT_ERR_INVALID_ARG, "codes_se or key_scale is NULL");
  if ((fmt->mant_bits > 0) != (codes_m != nullptr))
    return fail(POT_ERR_INVALID_ARG, "codes_m must be non-NULL exactly when mant_bits > 0");
  if (!aligned(codes_se, 16) || !aligned(key_scale, 4) || (codes_m && !aligned(codes_m, 8)))
    return fail(POT_ERR_INVALID_ARG, "misaligned codes_se / key_scale / codes_m");
  DecodeArgs a{};
  a.q = q;
  a.codes_se = codes_se;
  a.codes_m = codes_m;
  a.key_scale = key_scale;
  a.v8 = v_u8;
  a.v_exp = v_exp;
  a.out = out;
  a.frac_bits = fmt->frac_bits;
  a.hadamard = fmt->hadamard;
  return decode_common(engine == 0 ? kScorePot : kScoreDs4a, fmt->mant_bits, a, kv_head_of_q, B,
                       Hq, Hkv, T, t_cap, workspace, ws_bytes, dbg, stream, vf);
}

// Shared body of the 4-bit-value entry points; append: k_new and v_new are taken in.
pot_status decode_v4(bool append, const pot_format* fmt, int32_t engine, const float* q,
                     const uint16_t* k_new, const uint16_t* v_new, const uint8_t* codes_se,
                     const uint8_t* codes_m, const float* key_scale, const uint8_t* v_u4,
                     int64_t t_cap, const int32_t* seq_lens, const int32_t* kv_head_of_q,
                     int32_t B, int32_t Hq, int32_t Hkv, int32_t T, float* out, void* workspace,
                     size_t ws_bytes, pot_debug* dbg, void* stream) {
  pot_status st = check_format(fmt);
  if (st != POT_OK) return st;
  if (engine != 0 && engine != 1)
    return fail(POT_ERR_INVALID_ARG, "engine %d (0 shift-accumulate, 1 byte decode)", engine);
  if (engine == 1 && fmt->mant_bits != 0)
    return fail(POT_ERR_UNSUPPORTED, "the byte-decode path scores PoT-4 codes only (mant_bits 0)");
  if (append && (!k_new || !v_new)) return fail(POT_ERR_INVALID_ARG, "k_new or v_new is NULL");
  if (append && (!aligned(k_new, 16) || !aligned(v_new, 16)))
    return fail(POT_ERR_INVALID_ARG, "k_new and v_new must be 16-byte aligned");
  if (!codes_se || !key_scale) return fail(POT_ERR_INVALID_ARG, "codes_se or key_scale is NULL");
  if ((fmt->mant_bits > 0) != (codes_m != nullptr))
    return fail(POT_ERR_INVALID_ARG, "codes_m must be non-NULL exactly when mant_bits > 0");
  if (!aligned(codes_se, 16) || !aligned(key_scale, 4) || (codes_m && !aligned(codes_m, 8)))
    return fail(POT_ERR_INVALID_ARG, "misaligned codes_se / key_scale / codes_m");
  DecodeArgs a{};
  a.q = q;
  a.codes_se = codes_se;
  a.codes_m = codes_m;
  a.key_scale = key_scale;
  a.v4 = v_u4;
  a.seq_lens = seq_lens;
  a.out = out;
  a.frac_bits = fmt->frac_bits;
  a.hadamard = fmt->hadamard;
  if (append) {
    a.app_k = k_new;
    a.app_v = v_new;
    a.app_codes_se = const_cast<uint8_t*>(codes_se);
    a.app_codes_m = const_cast<uint8_t*>(codes_m);
    a.app_key_scale = const_cast<float*>(key_scale);
    a.app_v4 = const_cast<uint8_t*>(v_u4);
    a.app_tab = encode_tables(fmt->mant_bits);
  }
  return decode_common(engine == 0 ? kScorePot : kScoreDs4a, fmt->mant_bits, a, kv_head_of_q, B,
                       Hq, Hkv, T, t_cap, workspace, ws_bytes, dbg, stream, 3);
}

// Rows [t0, t0 + n_tok) of n_seq sequences of t_cap rows.
pot_status check_rows(int64_t n_seq, int64_t n_tok, int64_t t_cap, int64_t t0) {
  if (n_seq < 0 || n_tok < 0)
    return fail(POT_ERR_INVALID_ARG, "n_seq %lld / n_tok %lld < 0", (long long)n_seq,
                (long long)n_tok);
  if (t_cap < 8 || t_cap % 8)
    return fail(POT_ERR_INVALID_ARG, "t_cap %lld is not a positive multiple of 8",
                (long long)t_cap);
  if (t0 < 0 || n_tok > t_cap || t0 > t_cap - n_tok)
    return fail(POT_ERR_INVALID_ARG, "n_tok %lld tokens from %lld outside [0, t_cap = %lld)",
                (long long)n_tok, (long long)t0, (long long)t_cap);
  if (n_tok > 0 && n_seq > ((int64_t)1 << 30) / n_tok)
    return fail(POT_ERR_INVALID_ARG, "n_seq * n_tok too large");
  return POT_OK;
}

pot_status load_values(int format, const void* cache, const int8_t* v_exp, int64_t n_seq,
                       int64_t n_tok, int64_t t_cap, int64_t t0, uint16_t* v_fp16, void* stream) {
  pot_status st = check_rows(n_seq, n_tok, t_cap, t0);
  if (st != POT_OK) return st;
  if (n_seq == 0 || n_tok == 0) return ok();
  if (!cache || !v_fp16 || (format == 1 && !v_exp))
    return fail(POT_ERR_INVALID_ARG, "a value cache pointer or v_fp16 is NULL");
  if (!aligned(cache, 16) || !aligned(v_fp16, 16) || !aligned(v_exp, 16))
    return fail(POT_ERR_INVALID_ARG, "the value cache and v_fp16 must be 16-byte aligned");
  return hip_status(launch_load_values(format, cache, v_exp, n_seq, n_tok, t_cap, t0, v_fp16,
                                       static_cast<hipStream_t>(stream)),
                    "load values launch");
}

// One part of a projection and its output: both given, or neither.
pot_status check_part(const char* name, const pot_part& p, int32_t heads, int32_t B, int32_t S,
                      int size, RowsIn* in) {
  *in = RowsIn{};
  if (!p.rows) {
    if (p.out) return fail(POT_ERR_INVALID_ARG, "%s is left out, but not its output", name);
    return POT_OK;
  }
  if (!p.out) return fail(POT_ERR_INVALID_ARG, "%s has no output", name);
  if (heads < 1) return fail(POT_ERR_INVALID_ARG, "%d heads of %s", heads, name);
  const int64_t per16 = 16 / size;
  if (!aligned(p.rows, 16) || !aligned(p.out, 16) || !aligned(p.weight, 16) ||
      (B > 1 && p.stride_b % per16) || (S > 1 && p.stride_s % per16) ||
      (heads > 1 && p.stride_h % per16))
    return fail(POT_ERR_INVALID_ARG, "rows, weight and output of %s must be 16-byte aligned", name);
  *in = RowsIn{p.rows, B > 1 ? p.stride_b : 0, S > 1 ? p.stride_s : 0, heads > 1 ? p.stride_h : 0};
  return POT_OK;
}

// What pot_norm_rope and pot_paged_append check and pass on alike.
pot_status check_rope(const pot_rope& rope, int32_t dtype, int32_t weight_dtype, int32_t q_out_dtype,
                      float eps) {
  if (rope.head_dim != 64)
    return fail(POT_ERR_UNSUPPORTED, "head_dim %d (only 64)", rope.head_dim);
  const int r = rope.rot_dim;
  if (r < 0 || r > 64 || r % 2)
    return fail(POT_ERR_INVALID_ARG, "rot_dim %d (even, 0 .. 64)", r);
  if (rope.neighbours != 0 && rope.neighbours != 1)
    return fail(POT_ERR_INVALID_ARG, "neighbours %d (0 or 1)", rope.neighbours);
  if (rope.n_axes < 1 || rope.n_axes > POT_MAX_AXES)
    return fail(POT_ERR_INVALID_ARG, "n_axes %d (1 .. %d)", rope.n_axes, POT_MAX_AXES);
  for (int i = 0; i < r / 2; ++i)
    if (rope.axis_of_pair[i] >= rope.n_axes)
      return fail(POT_ERR_INVALID_ARG, "axis_of_pair[%d] = %d outside [0, %d)", i,
                  rope.axis_of_pair[i], rope.n_axes);
  for (const int32_t t : {dtype, weight_dtype, q_out_dtype})
    if (t < POT_FP16 || t > POT_FP32)
      return fail(POT_ERR_INVALID_ARG, "type %d (0 fp16, 1 bf16, 2 fp32)", t);
  if (!(eps >= 0.0f && eps <= 3.4e38f)) return fail(POT_ERR_INVALID_ARG, "eps %g", eps);
  return POT_OK;
}
void fill_rope(const pot_rope& rope, int32_t dtype, int32_t weight_dtype, int32_t q_out_dtype, float eps,
               NormRopeArgs* a) {
  a->eps = eps;
  a->dtype = dtype;
  a->weight_dtype = weight_dtype;
  a->q_out_dtype = q_out_dtype;
  a->rot_dim = rope.rot_dim;
  a->neighbours = rope.neighbours;
  a->n_axes = rope.n_axes;
  for (int i = 0; i < 32; ++i) a->axis_of_pair[i] = i < rope.rot_dim / 2 ? rope.axis_of_pair[i] : 0;
}

// A paged cache and the sequences of a call.
pot_status check_pages(const pot_format* fmt, const pot_pages* p, const int32_t* cu_new,
                       const int32_t* seq_lens, int32_t B, int32_t n, PagesArg* arg, PackedRows* rows) {
  if (!p) return fail(POT_ERR_INVALID_ARG, "pages is NULL");
  if (p->value_format != POT_VALUES_FP16 && p->value_format != POT_VALUES_INT4)
    return fail(POT_ERR_INVALID_ARG, "value_format %d (0 fp16, 1 4-bit)", p->value_format);
  if (p->Hkv < 1) return fail(POT_ERR_INVALID_ARG, "%d kv heads", p->Hkv);
  if (p->Hkv > kMaxHqArg) return fail(POT_ERR_UNSUPPORTED, "Hkv %d > %d", p->Hkv, kMaxHqArg);
  if (p->page_size < 8 || p->page_size % 8 || p->page_size > (1 << 24))
    return fail(POT_ERR_INVALID_ARG, "page_size %d is not a multiple of 8 up to 2^24", p->page_size);
  if (p->n_pages < 1 || p->table_len < 1)
    return fail(POT_ERR_INVALID_ARG, "n_pages %d or table_len %d < 1", p->n_pages, p->table_len);
  if ((int64_t)p->n_pages * p->Hkv > ((int64_t)1 << 33) / p->page_size)
    return fail(POT_ERR_INVALID_ARG, "n_pages * Hkv * page_size too large");
  if (B < 0 || n < 0) return fail(POT_ERR_INVALID_ARG, "B %d or n %d < 0", B, n);
  if (B > 65535) return fail(POT_ERR_UNSUPPORTED, "B %d > 65535", B);
  if (n > (1 << 23)) return fail(POT_ERR_UNSUPPORTED, "n %d > 2^23", n);
  if ((fmt->mant_bits > 0) != (p->codes_m != nullptr))
    return fail(POT_ERR_INVALID_ARG, "codes_m must be non-NULL exactly when mant_bits > 0");
  // without sequences the table and the lengths have no elements, and no address
  if (!p->codes_se || !p->key_scale || !p->values || (B > 0 && !p->table))
    return fail(POT_ERR_INVALID_ARG, "codes_se, key_scale, values or table is NULL");
  if (!aligned(p->codes_se, 16) || !aligned(p->codes_m, 8) || !aligned(p->key_scale, 16) ||
      !aligned(p->values, 16) || !aligned(p->table, 4))
    return fail(POT_ERR_INVALID_ARG, "misaligned codes_se / codes_m / key_scale / values / table");
  if (B > 0 && (!cu_new || !seq_lens))
    return fail(POT_ERR_INVALID_ARG, "cu_new or seq_lens is NULL");
  if (!aligned(cu_new, 4) || !aligned(seq_lens, 4))
    return fail(POT_ERR_INVALID_ARG, "cu_new and seq_lens must be 4-byte aligned");
  const uint32_t groups = (uint32_t)p->page_size / 8;
  *arg = PagesArg{p->codes_se, p->codes_m, p->key_scale, static_cast<uint8_t*>(p->values), p->table,
                  p->n_pages, p->Hkv, p->table_len, (int32_t)groups, page_div(groups)};
  *rows = PackedRows{cu_new, seq_lens, B, n};
  return POT_OK;
}

pot_status check_paged_sizes(int32_t B, int32_t n, int32_t Hq, int32_t Hkv, int32_t max_new,
                             int32_t max_len) {
  if (B < 0 || n < 0 || Hq < 1 || Hkv < 1 || max_new < 1 || max_len < 1)
    return fail(POT_ERR_INVALID_ARG, "bad sizes B=%d n=%d Hq=%d Hkv=%d max_new=%d max_len=%d", B, n, Hq, Hkv,
                max_new, max_len);
  if (B > 65535 || n > (1 << 23)) return fail(POT_ERR_UNSUPPORTED, "B %d > 65535 or n %d > 2^23", B, n);
  if (Hq > kMaxHqArg) return fail(POT_ERR_UNSUPPORTED, "Hq %d > %d", Hq, kMaxHqArg);
  if (Hq % Hkv) return fail(POT_ERR_UNSUPPORTED, "Hq %d not a multiple of Hkv %d", Hq, Hkv);
  if (max_len > kMaxKeys) return fail(POT_ERR_UNSUPPORTED, "max_len %d > %d", max_len, kMaxKeys);
  // a launch has fewer than 2^32 threads: 512 for 256 rows of a kv head, and for each sequence's last ones
  if ((int64_t)n * Hq / 256 + (int64_t)std::min(B, n) * Hkv >= (1 << 23) - kManyPieces)
    return fail(POT_ERR_UNSUPPORTED, "%d rows of %d heads in %d sequences of %d kv heads: too many for a launch", n, Hq, B,
                Hkv);
  return POT_OK;
}

// Head map with groups of any one size, [Hkv][G] a byte each.
pot_status check_head_groups(const int32_t* map, int Hq, int Hkv, uint32_t* q_of_kv) {
  if (!map) return fail(POT_ERR_INVALID_ARG, "kv_head_of_q is NULL");
  const int G = Hq / Hkv;
  int fill[kMaxHqArg] = {};
  for (int i = 0; i < Hq; ++i) {
    const int h = map[i];
    if (h < 0 || h >= Hkv)
      return fail(POT_ERR_INVALID_ARG, "kv_head_of_q[%d] = %d outside [0, %d)", i, h, Hkv);
    if (fill[h] >= G)
      return fail(POT_ERR_UNSUPPORTED, "kv head %d serves more than %d query heads", h, G);
    const int at = h * G + fill[h]++;
    q_of_kv[at >> 2] |= (uint32_t)i << (8 * (at & 3));
  }
  return POT_OK;
}

// How a paged attention call is split. A longer max_len never takes fewer splits than a shorter one or
// a window, so that the workspace of the former serves the latter.
PagedPlan paged_plan(int B, int n, int Hq, int Hkv, int max_new, int max_len, int window, int n_sink,
                     int mant_bits, bool uni, int value_format) {
  const int64_t G = Hq / Hkv, rows = std::min(max_new, n) * G;
  int64_t keys = max_len;  // that a row tile sees, at most
  if (window > 0) keys = std::min<int64_t>(keys, (int64_t)window + max_new + n_sink + 2 * kWTile);
  const int64_t tiles = (keys + kWTile - 1) / kWTile;
  PagedPlan p{};
  const bool few = rows <= kFewRows, many = !few;
  // one sequence, or all of them as long as they may be: nothing is left for the kernel of few rows
  const bool both = many && G <= kFewRows && B > 1 && n < (int64_t)B * max_new;
  if (few || both) {
    // 8 rows have a form of their own (64 single tokens on 4096 keys 24.1 us, by the form of 16 rows
    // 25.6); beside longer sequences those of 9 to 16 rows would go to the kernel of many for it
    p.few_limit = few && rows <= 8 ? 8 : kFewRows;
    // Ranges of at least 4 tiles; where there is a workgroup for every CU without a split, of so many
    // that the split repays its merge: 64 single tokens on 4096 keys of fp16 values 33 us in one range,
    // 38 in two; of 1024 keys of 4-bit values 10.7 and 14.6, of 8192 42 and 40, and with lengths from
    // 8192 down to 512 39 and 29.
    const int64_t units = (int64_t)B * Hkv;
    const int64_t most = units < 256 ? (tiles + 3) / 4 : tiles / (value_format == POT_VALUES_INT4 ? 32 : 64);
    const int per_cu = few_simd_waves(mant_bits, uni, p.few_limit == 8);
    p.few_splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>({256 * per_cu / units, most, 64}));
  }
  if (many) {
    p.many_rows = rows > 128 ? 256 : 128;  // 64 sequences of 16 tokens, 8 heads each: 46 us by 128, 54 by 256
    const int64_t R = p.many_rows, full = ((int64_t)n * G + R - 1) / R;
    p.many_tiles = (int64_t)n * G / R + std::min(B, n);
    // 512 rows of 8 heads on 8192 keys: 72 us with 512 pieces (two workgroups a CU), 92 with 256 or 1024
    if (full * Hkv < kManyPieces && tiles > kManyRange) p.many_extra = kManyPieces / Hkv;
  }
  return p;
}

struct PagedLayout {
  size_t many, pieces, total;
};
PagedLayout paged_layout(const PagedPlan& p, int B, int Hkv) {
  PagedLayout w{};
  if (p.few_splits > 1)
    w.many = align_up((size_t)B * Hkv * p.few_splits * kFewRows * kPartial * 4, 256);
  w.pieces = w.total = w.many;
  if (p.many_extra > 0) {
    const size_t n = (size_t)(p.many_tiles + p.many_extra);
    w.pieces += align_up(n * Hkv * p.many_rows * kPartial * 4, 256);
    w.total = w.pieces + align_up(n * sizeof(int4), 256);
  }
  return w;
}

}  // namespace

extern "C" {

const char* pot_status_string(pot_status s) {
  switch (s) {
    case POT_OK: return "POT_OK";
    case POT_ERR_INVALID_ARG: return "POT_ERR_INVALID_ARG";
    case POT_ERR_UNSUPPORTED: return "POT_ERR_UNSUPPORTED";
    case POT_ERR_WORKSPACE: return "POT_ERR_WORKSPACE";
    case POT_ERR_HIP: return "POT_ERR_HIP";
  }
  return "POT_ERR_UNKNOWN";
}

const char* pot_last_error(void) { return g_last_error.c_str(); }

size_t pot_code_bytes_per_row(const pot_format* fmt) {
  if (check_format(fmt) != POT_OK) return 0;
  return 32 + 8 * (size_t)fmt->mant_bits;
}

pot_status pot_encode_keys(const pot_format* fmt, const uint16_t* k_fp16, int64_t n_rows,
                           int64_t out_row_stride, int32_t scale_mode, float* key_scale,
                           uint8_t* codes_se, uint8_t* codes_m, void* stream) {
  pot_status st = check_format(fmt);
  if (st != POT_OK) return st;
  if (n_rows < 0) return fail(POT_ERR_INVALID_ARG, "n_rows %lld < 0", (long long)n_rows);
  if (out_row_stride < 1)
    return fail(POT_ERR_INVALID_ARG, "out_row_stride %lld < 1", (long long)out_row_stride);
  if (scale_mode != 0 && scale_mode != 1)
    return fail(POT_ERR_INVALID_ARG, "scale_mode %d (0 or 1)", scale_mode);
  if (n_rows == 0) return ok();
  if (!k_fp16 || !key_scale || !codes_se)
    return fail(POT_ERR_INVALID_ARG, "k_fp16, key_scale or codes_se is NULL");
  if ((fmt->mant_bits > 0) != (codes_m != nullptr))
    return fail(POT_ERR_INVALID_ARG, "codes_m must be non-NULL exactly when mant_bits > 0");
  if (!aligned(k_fp16, 16) || !aligned(codes_se, 16) || !aligned(key_scale, 4) ||
      (codes_m && !aligned(codes_m, 8)))
    return fail(POT_ERR_INVALID_ARG, "misaligned k_fp16 / codes_se / key_scale / codes_m");
  if (n_rows > (int64_t)1 << 36) return fail(POT_ERR_INVALID_ARG, "n_rows too large");
  const EncodeTables& tab = encode_tables(fmt->mant_bits);
  return hip_status(launch_encode_pot(k_fp16, n_rows, out_row_stride, scale_mode, fmt->hadamard,
                                      key_scale, codes_se, codes_m, tab,
                                      static_cast<hipStream_t>(stream)),
                    "encode launch");
}

pot_status pot_store_values(const uint16_t* v_fp16, int64_t n_seq, int64_t n_tok, int64_t t_cap,
                            int64_t t0, uint16_t* v_cache, void* stream) {
  if (n_seq < 0 || n_tok < 0)
    return fail(POT_ERR_INVALID_ARG, "n_seq %lld / n_tok %lld < 0", (long long)n_seq,
                (long long)n_tok);
  if (t_cap < 8 || t_cap % 8)
    return fail(POT_ERR_INVALID_ARG, "t_cap %lld is not a positive multiple of 8",
                (long long)t_cap);
  if (t0 < 0 || t0 + n_tok > t_cap)
    return fail(POT_ERR_INVALID_ARG, "tokens [%lld, %lld) outside [0, t_cap = %lld)",
                (long long)t0, (long long)(t0 + n_tok), (long long)t_cap);
  if (n_seq == 0 || n_tok == 0) return ok();
  if (!v_fp16 || !v_cache) return fail(POT_ERR_INVALID_ARG, "v_fp16 or v_cache is NULL");
  if (!aligned(v_fp16, 16) || !aligned(v_cache, 16))
    return fail(POT_ERR_INVALID_ARG, "v_fp16 and v_cache must be 16-byte aligned");
  return hip_status(launch_store_values(v_fp16, n_seq, n_tok, t_cap, t0, v_cache,
                                        static_cast<hipStream_t>(stream)),
                    "store values launch");
}

pot_status pot_store_values_int8(const uint16_t* v_fp16, int64_t n_seq, int64_t n_tok,
                                 int64_t t_cap, int64_t t0, uint8_t* v_u8, int8_t* v_exp,
                                 void* stream) {
  if (n_seq < 0 || n_tok < 0)
    return fail(POT_ERR_INVALID_ARG, "n_seq %lld / n_tok %lld < 0", (long long)n_seq,
                (long long)n_tok);
  if (t_cap < 8 || t_cap % 8)
    return fail(POT_ERR_INVALID_ARG, "t_cap %lld is not a positive multiple of 8",
                (long long)t_cap);
  if (t0 < 0 || t0 + n_tok > t_cap)
    return fail(POT_ERR_INVALID_ARG, "tokens [%lld, %lld) outside [0, t_cap = %lld)",
                (long long)t0, (long long)(t0 + n_tok), (long long)t_cap);
  if (n_seq == 0 || n_tok == 0) return ok();
  if (!v_fp16 || !v_u8 || !v_exp)
    return fail(POT_ERR_INVALID_ARG, "v_fp16, v_u8 or v_exp is NULL");
  if (!aligned(v_fp16, 16) || !aligned(v_u8, 16) || !aligned(v_exp, 16))
    return fail(POT_ERR_INVALID_ARG, "v_fp16, v_u8 and v_exp must be 16-byte aligned");
  if (n_seq > ((int64_t)1 << 31) / n_tok)
    return fail(POT_ERR_INVALID_ARG, "n_seq * n_tok too large");
  return hip_status(launch_store_values_i8(v_fp16, n_seq, n_tok, t_cap, t0, v_u8, v_exp,
                                           static_cast<hipStream_t>(stream)),
                    "store values launch");
}

pot_status pot_store_values_int4(const uint16_t* v_fp16, int64_t n_seq, int64_t n_tok,
                                 int64_t t_cap, int64_t t0, uint8_t* v_u4, void* stream) {
  pot_status st = check_rows(n_seq, n_tok, t_cap, t0);
  if (st != POT_OK) return st;
  if (n_seq == 0 || n_tok == 0) return ok();
  if (!v_fp16 || !v_u4) return fail(POT_ERR_INVALID_ARG, "v_fp16 or v_u4 is NULL");
  if (!aligned(v_fp16, 16) || !aligned(v_u4, 16))
    return fail(POT_ERR_INVALID_ARG, "v_fp16 and v_u4 must be 16-byte aligned");
  return hip_status(launch_store_values_i4(v_fp16, n_seq, n_tok, t_cap, t0, v_u4,
                                           static_cast<hipStream_t>(stream)),
                    "store values launch");
}

pot_status pot_load_keys(const pot_format* fmt, const uint8_t* codes_se, const uint8_t* codes_m,
                         const float* key_scale, int64_t n_seq, int64_t n_tok, int64_t t_cap,
                         int64_t t0, uint16_t* k_fp16, void* stream) {
  pot_status st = check_format(fmt);
  if (st != POT_OK) return st;
  st = check_rows(n_seq, n_tok, t_cap, t0);
  if (st != POT_OK) return st;
  if (n_seq == 0 || n_tok == 0) return ok();
  if (!codes_se || !key_scale || !k_fp16)
    return fail(POT_ERR_INVALID_ARG, "codes_se, key_scale or k_fp16 is NULL");
  if ((fmt->mant_bits > 0) != (codes_m != nullptr))
    return fail(POT_ERR_INVALID_ARG, "codes_m must be non-NULL exactly when mant_bits > 0");
  if (!aligned(codes_se, 16) || !aligned(key_scale, 4) || !aligned(k_fp16, 16) ||
      (codes_m && !aligned(codes_m, 8)))
    return fail(POT_ERR_INVALID_ARG, "misaligned codes_se / key_scale / codes_m / k_fp16");
  return hip_status(launch_load_keys(fmt->mant_bits, fmt->hadamard, codes_se, codes_m, key_scale,
                                     n_seq, n_tok, t_cap, t0, k_fp16,
                                     static_cast<hipStream_t>(stream)),
                    "load keys launch");
}

pot_status pot_load_values(const uint16_t* v_cache, int64_t n_seq, int64_t n_tok, int64_t t_cap,
                           int64_t t0, uint16_t* v_fp16, void* stream) {
  return load_values(0, v_cache, nullptr, n_seq, n_tok, t_cap, t0, v_fp16, stream);
}

pot_status pot_load_values_int8(const uint8_t* v_u8, const int8_t* v_exp, int64_t n_seq,
                                int64_t n_tok, int64_t t_cap, int64_t t0, uint16_t* v_fp16,
                                void* stream) {
  return load_values(1, v_u8, v_exp, n_seq, n_tok, t_cap, t0, v_fp16, stream);
}

pot_status pot_load_values_int4(const uint8_t* v_u4, int64_t n_seq, int64_t n_tok, int64_t t_cap,
                                int64_t t0, uint16_t* v_fp16, void* stream) {
  return load_values(2, v_u4, nullptr, n_seq, n_tok, t_cap, t0, v_fp16, stream);
}

pot_status pot_norm_rope(const pot_rope* rope, int32_t dtype, const pot_part* parts,
                         int32_t weight_dtype, float eps, const int64_t* positions,
                         const double* inv_freq, int32_t B, int32_t S, int32_t Hq, int32_t Hkv,
                         int32_t q_out_dtype, void* stream) {
  if (!rope || !parts) return fail(POT_ERR_INVALID_ARG, "rope or parts is NULL");
  pot_status st = check_rope(*rope, dtype, weight_dtype, q_out_dtype, eps);
  if (st != POT_OK) return st;
  const int r = rope->rot_dim;
  if (B < 0 || S < 0 || Hq < 0 || Hkv < 0)
    return fail(POT_ERR_INVALID_ARG, "bad shape B=%d S=%d Hq=%d Hkv=%d", B, S, Hq, Hkv);
  if (Hq > 1024 || Hkv > 1024)
    return fail(POT_ERR_UNSUPPORTED, "%d and %d heads (at most 1024)", Hq, Hkv);
  if (B == 0 || S == 0) return ok();
  NormRopeArgs a{};
  const int size = dtype == POT_FP32 ? 4 : 2;
  st = check_part("q", parts[0], Hq, B, S, size, &a.q);
  if (st == POT_OK) st = check_part("k", parts[1], Hkv, B, S, size, &a.k);
  if (st == POT_OK) st = check_part("v", parts[2], Hkv, B, S, size, &a.v);
  if (st != POT_OK) return st;
  if (parts[2].weight) return fail(POT_ERR_INVALID_ARG, "v takes no weight");
  if (!a.q.data && !a.k.data && !a.v.data) return ok();
  if (r > 0 && (a.q.data || a.k.data) && (!positions || !inv_freq))
    return fail(POT_ERR_INVALID_ARG, "positions or inv_freq is NULL");
  if (!aligned(positions, 8) || !aligned(inv_freq, 8))
    return fail(POT_ERR_INVALID_ARG, "positions and inv_freq must be 8-byte aligned");
  if ((int64_t)B * S > ((int64_t)1 << 28))  // 2^31 work-items, of 2^32 that a dispatch holds
    return fail(POT_ERR_INVALID_ARG, "B * S too large");
  a.q_weight = a.q.data ? parts[0].weight : nullptr;
  a.k_weight = a.k.data ? parts[1].weight : nullptr;
  a.positions = positions;
  a.inv_freq = inv_freq;
  a.q_out = parts[0].out;
  a.k_out = static_cast<uint16_t*>(parts[1].out);
  a.v_out = static_cast<uint16_t*>(parts[2].out);
  a.B = B;
  a.S = S;
  a.Hq = a.q.data ? Hq : 0;
  a.Hkv = a.k.data || a.v.data ? Hkv : 0;
  fill_rope(*rope, dtype, weight_dtype, q_out_dtype, eps, &a);
  return hip_status(launch_norm_rope(a, static_cast<hipStream_t>(stream)), "norm and rotation launch");
}

pot_status pot_paged_append(const pot_format* fmt, const pot_rope* rope, int32_t dtype,
                            const pot_part* parts, int32_t weight_dtype, float eps,
                            const int64_t* positions, const double* inv_freq,
                            const pot_pages* pages, const int32_t* cu_new,
                            const int32_t* seq_lens, int32_t B, int32_t n, int32_t Hq,
                            int32_t q_out_dtype, void* stream) {
  pot_status st = check_format(fmt);
  if (st != POT_OK) return st;
  if (!rope || !parts) return fail(POT_ERR_INVALID_ARG, "rope or parts is NULL");
  st = check_rope(*rope, dtype, weight_dtype, q_out_dtype, eps);
  if (st != POT_OK) return st;
  PagedAppendArgs a{};
  st = check_pages(fmt, pages, cu_new, seq_lens, B, n, &a.pages, &a.packed);
  if (st != POT_OK) return st;
  if (Hq < 0 || Hq > 1024) return fail(POT_ERR_UNSUPPORTED, "%d query heads (0 .. 1024)", Hq);
  if (B == 0 || n == 0) return ok();
  const int size = dtype == POT_FP32 ? 4 : 2, per16 = 16 / size;
  NormRopeArgs& r = a.rows;
  for (int i = 0; i < 3; ++i) {
    static const char* const kName[3] = {"q", "k", "v"};
    const pot_part& p = parts[i];
    const int heads = i == 0 ? Hq : pages->Hkv;
    if (i == 0 && !p.rows) {
      if (p.out) return fail(POT_ERR_INVALID_ARG, "q is left out, but not its output");
      continue;
    }
    if (!p.rows) return fail(POT_ERR_INVALID_ARG, "%s is NULL", kName[i]);
    if (heads < 1) return fail(POT_ERR_INVALID_ARG, "%d heads of q", heads);
    if ((i == 0) != (p.out != nullptr))
      return fail(POT_ERR_INVALID_ARG, i == 0 ? "q has no output" : "%s goes into the pages: its out is NULL",
                  kName[i]);
    if (!aligned(p.rows, 16) || !aligned(p.out, 16) || !aligned(p.weight, 16) ||
        (n > 1 && p.stride_s % per16) || (heads > 1 && p.stride_h % per16))
      return fail(POT_ERR_INVALID_ARG, "rows, weight and output of %s must be 16-byte aligned", kName[i]);
    (i == 0 ? r.q : i == 1 ? r.k : r.v) =
        RowsIn{p.rows, 0, n > 1 ? p.stride_s : 0, heads > 1 ? p.stride_h : 0};
  }
  if (parts[2].weight) return fail(POT_ERR_INVALID_ARG, "v takes no weight");
  if (rope->rot_dim > 0 && !inv_freq) return fail(POT_ERR_INVALID_ARG, "inv_freq is NULL");
  if (!aligned(positions, 8) || !aligned(inv_freq, 8))
    return fail(POT_ERR_INVALID_ARG, "positions and inv_freq must be 8-byte aligned");
  r.q_weight = r.q.data ? parts[0].weight : nullptr;
  r.k_weight = parts[1].weight;
  r.positions = positions;
  r.inv_freq = inv_freq;
  r.q_out = parts[0].out;
  r.B = 1;
  r.S = n;
  r.Hq = r.q.data ? Hq : 0;
  r.Hkv = pages->Hkv;
  fill_rope(*rope, dtype, weight_dtype, q_out_dtype, eps, &r);
  a.tab = encode_tables(fmt->mant_bits);
  a.hadamard = fmt->hadamard;
  a.value_format = pages->value_format;
  return hip_status(launch_paged_append(a, static_cast<hipStream_t>(stream)), "paged append launch");
}

size_t pot_paged_workspace_bytes(int32_t B, int32_t n, int32_t Hq, int32_t Hkv, int32_t max_new,
                                 int32_t max_len) {
  if (check_paged_sizes(B, n, Hq, Hkv, max_new, max_len) != POT_OK) return 0;
  if (B == 0 || n == 0) return 0;
  return paged_layout(paged_plan(B, n, Hq, Hkv, max_new, max_len, 0, 0, 0, true, POT_VALUES_INT4), B, Hkv).total;
}

pot_status pot_paged_attention(const pot_format* fmt, int32_t dtype, const void* q,
                               int64_t stride_t, int64_t stride_h, const pot_pages* pages,
                               const int32_t* cu_new, const int32_t* seq_lens,
                               const int32_t* kv_head_of_q, int32_t B, int32_t n, int32_t Hq,
                               int32_t max_new, int32_t max_len, int32_t window, int32_t n_sink,
                               int32_t out_dtype, void* out, void* workspace, size_t ws_bytes,
                               void* stream) {
  pot_status st = check_format(fmt);
  if (st != POT_OK) return st;
  for (const int32_t t : {dtype, out_dtype})
    if (t < POT_FP16 || t > POT_FP32)
      return fail(POT_ERR_INVALID_ARG, "type %d (0 fp16, 1 bf16, 2 fp32)", t);
  PagedAttendArgs a{};
  st = check_pages(fmt, pages, cu_new, seq_lens, B, n, &a.pages, &a.packed);
  if (st == POT_OK) st = check_paged_sizes(B, n, Hq, pages->Hkv, max_new, max_len);
  if (st != POT_OK) return st;
  if (max_len > (int64_t)pages->table_len * pages->page_size)
    return fail(POT_ERR_INVALID_ARG, "max_len %d > %d pages of %d", max_len, pages->table_len, pages->page_size);
  if (window < 0 || n_sink < 0)
    return fail(POT_ERR_INVALID_ARG, "window %d or n_sink %d < 0", window, n_sink);
  st = check_head_groups(kv_head_of_q, Hq, pages->Hkv, a.q_of_kv);
  if (st != POT_OK) return st;
  if (B == 0 || n == 0) return ok();
  if (!q || !out) return fail(POT_ERR_INVALID_ARG, "q or out is NULL");
  const int per16 = dtype == POT_FP32 ? 4 : 8;
  if (!aligned(q, 16) || !aligned(out, 16) || (n > 1 && stride_t % per16) || (Hq > 1 && stride_h % per16))
    return fail(POT_ERR_INVALID_ARG, "q's rows and out must be 16-byte aligned");
  // past the longest sequence a window takes nothing off
  a.window = window >= (1 << 24) ? 0 : window;
  a.n_sink = std::min(n_sink, 1 << 24);
  a.plan = paged_plan(B, n, Hq, pages->Hkv, max_new, max_len, a.window, a.n_sink,
                      fmt->mant_bits, pages->page_size % kWTile == 0, pages->value_format);
  const PagedLayout w = paged_layout(a.plan, B, pages->Hkv);
  if (w.total > 0 && !workspace) return fail(POT_ERR_INVALID_ARG, "workspace is NULL");
  if (!aligned(workspace, 256))
    return fail(POT_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  if (ws_bytes < w.total)
    return fail(POT_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, w.total);
  a.q = q;
  a.q_stride_t = n > 1 ? stride_t : 0;
  a.q_stride_h = Hq > 1 ? stride_h : 0;
  a.out = out;
  a.few_part = static_cast<float*>(workspace);
  a.many_part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + w.many);
  a.many_pieces = reinterpret_cast<int4*>(static_cast<uint8_t*>(workspace) + w.pieces);
  a.Hq = Hq;
  a.G = Hq / pages->Hkv;
  a.max_new = max_new;
  a.max_len = max_len;
  a.dtype = dtype;
  a.out_dtype = out_dtype;
  a.hadamard = fmt->hadamard;
  a.mant_bits = fmt->mant_bits;
  a.value_format = pages->value_format;
  hipError_t e = hipSuccess;
  if (a.plan.many_tiles > 0) e = launch_paged_many(a, static_cast<hipStream_t>(stream));
  if (e == hipSuccess && a.plan.few_splits > 0) e = launch_paged_few(a, static_cast<hipStream_t>(stream));
  return hip_status(e, "paged attention launch");
}

size_t pot_decode_workspace_bytes(int32_t B, int32_t Hq, int32_t Hkv, int32_t T) {
  if (!shape_ok(B, Hq, Hkv, T)) return 0;
  return ws_layout(B, Hq, Hkv, plan_bound(B, Hkv, T).n_splits).total;
}

size_t pot_decode_workspace_bytes_for_splits(int32_t B, int32_t Hq, int32_t Hkv, int32_t T,
                                             int32_t n_splits) {
  if (!shape_ok(B, Hq, Hkv, T) || n_splits < 0) return 0;
  const Plan p = n_splits > 0 ? plan_from_count(T, n_splits) : plan_bound(B, Hkv, T);
  return ws_layout(B, Hq, Hkv, p.n_splits).total;
}

pot_status pot_workspace_init(void* workspace, size_t ws_bytes, void* stream) {
  if (!workspace) return fail(POT_ERR_INVALID_ARG, "workspace is NULL");
  return hip_status(launch_fill_zero(workspace, ws_bytes, static_cast<hipStream_t>(stream)),
                    "workspace init");
}

pot_status pot_decode_attention(const pot_format* fmt, const float* q, const uint8_t* codes_se,
                                const uint8_t* codes_m, const float* key_scale,
                                const uint16_t* v_cache, int64_t t_cap,
                                const int32_t* kv_head_of_q, int32_t B, int32_t Hq, int32_t Hkv,
                                int32_t T, float* out, void* workspace, size_t ws_bytes,
                                pot_debug* dbg, void* stream) {
  pot_status st = check_format(fmt);
  if (st != POT_OK) return st;
  if (!codes_se || !key_scale) return fail(POT_ERR_INVALID_ARG, "codes_se or key_scale is NULL");
  if ((fmt->mant_bits > 0) != (codes_m != nullptr))
    return fail(POT_ERR_INVALID_ARG, "codes_m must be non-NULL exactly when mant_bits > 0");
  if (!aligned(codes_se, 16) || !aligned(key_scale, 4) || (codes_m && !aligned(codes_m, 8)))
    return fail(POT_ERR_INVALID_ARG, "misaligned codes_se / key_scale / codes_m");
  DecodeArgs a{};
  a.q = q;
  a.codes_se = codes_se;
  a.codes_m = codes_m;
  a.key_scale = key_scale;
  a.v = v_cache;
  a.out = out;
  a.frac_bits = fmt->frac_bits;
  a.hadamard = fmt->hadamard;
  return decode_common(kScorePot, fmt->mant_bits, a, kv_head_of_q, B, Hq, Hkv, T, t_cap,
                       workspace, ws_bytes, dbg, stream);
}

pot_status pot_append_decode_attention(const pot_format* fmt, const float* q,
                                       const uint16_t* k_new, const uint16_t* v_new,
                                       uint8_t* codes_se, uint8_t* codes_m, float* key_scale,
                                       uint16_t* v_cache, int64_t t_cap,
                                       const int32_t* kv_head_of_q, int32_t B, int32_t Hq,
                                       int32_t Hkv, int32_t T, float* out, void* workspace,
                                       size_t ws_bytes, pot_debug* dbg, void* stream) {
  pot_status st = check_format(fmt);
  if (st != POT_OK) return st;
  if (!k_new || !v_new) return fail(POT_ERR_INVALID_ARG, "k_new or v_new is NULL");
  if (!aligned(k_new, 16) || !aligned(v_new, 16))
    return fail(POT_ERR_INVALID_ARG, "k_new and v_new must be 16-byte aligned");
  if (!codes_se || !key_scale) return fail(POT_ERR_INVALID_ARG, "codes_se or key_scale is NULL");
  if ((fmt->mant_bits > 0) != (codes_m != nullptr))
    return fail(POT_ERR_INVALID_ARG, "codes_m must be non-NULL exactly when mant_bits > 0");
  if (!aligned(codes_se, 16) || !aligned(key_scale, 4) || (codes_m && !aligned(codes_m, 8)))
    return fail(POT_ERR_INVALID_ARG, "misaligned codes_se / key_scale / codes_m");
  DecodeArgs a{};
  a.q = q;
  a.codes_se = codes_se;
  a.codes_m = codes_m;
  a.key_scale = key_scale;
  a.v = v_cache;
  a.out = out;
  a.frac_bits = fmt->frac_bits;
  a.hadamard = fmt->hadamard;
  a.app_k = k_new;
  a.app_v = v_new;
  a.app_codes_se = codes_se;
  a.app_codes_m = codes_m;
  a.app_key_scale = key_scale;
  a.app_v_cache = v_cache;
  a.app_tab = encode_tables(fmt->mant_bits);
  return decode_common(kScorePot, fmt->mant_bits, a, kv_head_of_q, B, Hq, Hkv, T, t_cap,
                       workspace, ws_bytes, dbg, stream);
}

pot_status pot_decode_attention_v8(const pot_format* fmt, int32_t engine, const float* q,
                                   const uint8_t* codes_se, const uint8_t* codes_m,
                                   const float* key_scale, const uint8_t* v_u8,
                                   const int8_t* v_exp, int64_t t_cap,
                                   const int32_t* kv_head_of_q, int32_t B, int32_t Hq,
                                   int32_t Hkv, int32_t T, float* out, void* workspace,
                                   size_t ws_bytes, pot_debug* dbg, void* stream) {
  return decode_v8(1, fmt, engine, q, codes_se, codes_m, key_scale, v_u8, v_exp, t_cap,
                   kv_head_of_q, B, Hq, Hkv, T, out, workspace, ws_bytes, dbg, stream);
}

pot_status pot_decode_attention_v8_pow2(const pot_format* fmt, int32_t engine, const float* q,
                                        const uint8_t* codes_se, const uint8_t* codes_m,
                                        const float* key_scale, const uint8_t* v_u8,
                                        const int8_t* v_exp, int64_t t_cap,
                                        const int32_t* kv_head_of_q, int32_t B, int32_t Hq,
                                        int32_t Hkv, int32_t T, float* out, void* workspace,
                                        size_t ws_bytes, pot_debug* dbg, void* stream) {
  return decode_v8(2, fmt, engine, q, codes_se, codes_m, key_scale, v_u8, v_exp, t_cap,
                   kv_head_of_q, B, Hq, Hkv, T, out, workspace, ws_bytes, dbg, stream);
}

pot_status pot_append_decode_attention_v8(const pot_format* fmt, int32_t engine,
                                          const float* q, const uint16_t* k_new,
                                          const uint16_t* v_new, uint8_t* codes_se,
                                          uint8_t* codes_m, float* key_scale, uint8_t* v_u8,
                                          int8_t* v_exp, int64_t t_cap,
                                          const int32_t* kv_head_of_q, int32_t B, int32_t Hq,
                                          int32_t Hkv, int32_t T, float* out, void* workspace,
                                          size_t ws_bytes, pot_debug* dbg, void* stream) {
  pot_status st = check_format(fmt);
  if (st != POT_OK) return st;
  if (engine != 0 && engine != 1)
    return fail(POT_ERR_INVALID_ARG, "engine %d (0 shift-accumulate, 1 byte decode)", engine);
  if (engine == 1 && fmt->mant_bits != 0)
    return fail(POT_ERR_UNSUPPORTED, "the byte-decode path scores PoT-4 codes only (mant_bits 0)");
  if (!k_new || !v_new) return fail(POT_ERR_INVALID_ARG, "k_new or v_new is NULL");
  if (!aligned(k_new, 16) || !aligned(v_new, 16))
    return fail(POT_ERR_INVALID_ARG, "k_new and v_new must be 16-byte aligned");
  if (!codes_se || !key_scale) return fail(POT_ERR_INVALID_ARG, "codes_se or key_scale is NULL");
  if ((fmt->mant_bits > 0) != (codes_m != nullptr))
    return fail(POT_ERR_INVALID_ARG, "codes_m must be non-NULL exactly when mant_bits > 0");
  if (!aligned(codes_se, 16) || !aligned(key_scale, 4) || (codes_m && !aligned(codes_m, 8)))
    return fail(POT_ERR_INVALID_ARG, "misaligned codes_se / key_scale / codes_m");
  DecodeArgs a{};
  a.q = q;
  a.codes_se = codes_se;
  a.codes_m = codes_m;
  a.key_scale = key_scale;
  a.v8 = v_u8;
  a.v_exp = v_exp;
  a.out = out;
  a.frac_bits = fmt->frac_bits;
  a.hadamard = fmt->hadamard;
  a.app_k = k_new;
  a.app_v = v_new;
  a.app_codes_se = codes_se;
  a.app_codes_m = codes_m;
  a.app_key_scale = key_scale;
  a.app_v8 = v_u8;
  a.app_v_exp = v_exp;
  a.app_tab = encode_tables(fmt->mant_bits);
  return decode_common(engine == 0 ? kScorePot : kScoreDs4a, fmt->mant_bits, a, kv_head_of_q, B,
                       Hq, Hkv, T, t_cap, workspace, ws_bytes, dbg, stream, 1);
}

pot_status pot_decode_attention_v4(const pot_format* fmt, int32_t engine, const float* q,
                                   const uint8_t* codes_se, const uint8_t* codes_m,
                                   const float* key_scale, const uint8_t* v_u4, int64_t t_cap,
                                   const int32_t* seq_lens, const int32_t* kv_head_of_q, int32_t B,
                                   int32_t Hq, int32_t Hkv, int32_t T, float* out, void* workspace,
                                   size_t ws_bytes, pot_debug* dbg, void* stream) {
  return decode_v4(false, fmt, engine, q, nullptr, nullptr, codes_se, codes_m, key_scale, v_u4,
                   t_cap, seq_lens, kv_head_of_q, B, Hq, Hkv, T, out, workspace, ws_bytes, dbg,
                   stream);
}

pot_status pot_append_decode_attention_v4(const pot_format* fmt, int32_t engine, const float* q,
                                          const uint16_t* k_new, const uint16_t* v_new,
                                          uint8_t* codes_se, uint8_t* codes_m, float* key_scale,
                                          uint8_t* v_u4, int64_t t_cap, const int32_t* seq_lens,
                                          const int32_t* kv_head_of_q, int32_t B, int32_t Hq,
                                          int32_t Hkv, int32_t T, float* out, void* workspace,
                                          size_t ws_bytes, pot_debug* dbg, void* stream) {
  return decode_v4(true, fmt, engine, q, k_new, v_new, codes_se, codes_m, key_scale, v_u4, t_cap,
                   seq_lens, kv_head_of_q, B, Hq, Hkv, T, out, workspace, ws_bytes, dbg, stream);
}

pot_status pot_ds4a_decode_attention(const pot_format* fmt, const float* q,
                                     const uint8_t* codes_se, const float* key_scale,
                                     const uint16_t* v_cache, int64_t t_cap,
                                     const int32_t* kv_head_of_q, int32_t B, int32_t Hq,
                                     int32_t Hkv, int32_t T, float* out, void* workspace,
                                     size_t ws_bytes, pot_debug* dbg, void* stream) {
  pot_status st = check_format(fmt);
  if (st != POT_OK) return st;
  if (fmt->mant_bits != 0)
    return fail(POT_ERR_UNSUPPORTED, "the byte-decode path scores PoT-4 codes only (mant_bits 0)");
  if (!codes_se || !key_scale) return fail(POT_ERR_INVALID_ARG, "codes_se or key_scale is NULL");
  if (!aligned(codes_se, 16) || !aligned(key_scale, 4))
    return fail(POT_ERR_INVALID_ARG, "misaligned codes_se / key_scale");
  DecodeArgs a{};
  a.q = q;
  a.codes_se = codes_se;
  a.key_scale = key_scale;
  a.v = v_cache;
  a.out = out;
  a.frac_bits = fmt->frac_bits;
  a.hadamard = fmt->hadamard;
  return decode_common(kScoreDs4a, 0, a, kv_head_of_q, B, Hq, Hkv, T, t_cap, workspace, ws_bytes,
                       dbg, stream);
}

pot_status pot_dot_decode_attention(const pot_format* fmt, const float* q,
                                    const uint8_t* codes_se, const uint8_t* codes_m,
                                    const float* key_scale, const uint16_t* v_cache,
                                    int64_t t_cap, const int32_t* kv_head_of_q, int32_t B,
                                    int32_t Hq, int32_t Hkv, int32_t T, float* out,
                                    void* workspace, size_t ws_bytes, pot_debug* dbg,
                                    void* stream) {
  pot_status st = check_format(fmt);
  if (st != POT_OK) return st;
  if (!codes_se || !key_scale) return fail(POT_ERR_INVALID_ARG, "codes_se or key_scale is NULL");
  if ((fmt->mant_bits > 0) != (codes_m != nullptr))
    return fail(POT_ERR_INVALID_ARG, "codes_m must be non-NULL exactly when mant_bits > 0");
  if (!aligned(codes_se, 16) || !aligned(key_scale, 4) || (codes_m && !aligned(codes_m, 8)))
    return fail(POT_ERR_INVALID_ARG, "misaligned codes_se / key_scale / codes_m");
  DecodeArgs a{};
  a.q = q;
  a.codes_se = codes_se;
  a.codes_m = codes_m;
  a.key_scale = key_scale;
  a.v = v_cache;
  a.out = out;
  a.frac_bits = fmt->frac_bits;
  a.hadamard = fmt->hadamard;
  return decode_common(kScoreDs4a, fmt->mant_bits, a, kv_head_of_q, B, Hq, Hkv, T, t_cap,
                       workspace, ws_bytes, dbg, stream);
}

pot_status pot_int8_encode_keys(const uint16_t* k_fp16, int64_t n_rows, int64_t out_row_stride,
                                int32_t hadamard, float* key_scale, int8_t* codes, void* stream) {
  if (n_rows < 0) return fail(POT_ERR_INVALID_ARG, "n_rows %lld < 0", (long long)n_rows);
  if (out_row_stride < 1)
    return fail(POT_ERR_INVALID_ARG, "out_row_stride %lld < 1", (long long)out_row_stride);
  if (hadamard != 0 && hadamard != 1)
    return fail(POT_ERR_INVALID_ARG, "hadamard %d (0 or 1)", hadamard);
  if (n_rows == 0) return ok();
  if (!k_fp16 || !key_scale || !codes)
    return fail(POT_ERR_INVALID_ARG, "k_fp16, key_scale or codes is NULL");
  if (!aligned(k_fp16, 16) || !aligned(codes, 16) || !aligned(key_scale, 4))
    return fail(POT_ERR_INVALID_ARG, "misaligned k_fp16 / codes / key_scale");
  return hip_status(launch_encode_int8(k_fp16, n_rows, out_row_stride, hadamard, key_scale,
                                       codes, static_cast<hipStream_t>(stream)),
                    "int8 encode launch");
}

pot_status pot_int8_decode_attention(const float* q, const int8_t* codes, const float* key_scale,
                                     const uint16_t* v_cache, int64_t t_cap,
                                     const int32_t* kv_head_of_q, int32_t B, int32_t Hq,
                                     int32_t Hkv, int32_t T, int32_t hadamard, float* out,
                                     void* workspace, size_t ws_bytes, pot_debug* dbg,
                                     void* stream) {
  if (hadamard != 0 && hadamard != 1)
    return fail(POT_ERR_INVALID_ARG, "hadamard %d (0 or 1)", hadamard);
  if (!codes || !key_scale) return fail(POT_ERR_INVALID_ARG, "codes or key_scale is NULL");
  if (!aligned(codes, 16) || !aligned(key_scale, 4))
    return fail(POT_ERR_INVALID_ARG, "misaligned codes / key_scale");
  DecodeArgs a{};
  a.q = q;
  a.codes_i8 = codes;
  a.key_scale = key_scale;
  a.v = v_cache;
  a.out = out;
  a.hadamard = hadamard;
  return decode_common(kScoreInt8, 0, a, kv_head_of_q, B, Hq, Hkv, T, t_cap, workspace, ws_bytes,
                       dbg, stream);
}

pot_status pot_fp16_decode_attention(const float* q, const uint16_t* k_fp16,
                                     const uint16_t* v_cache, int64_t t_cap,
                                     const int32_t* kv_head_of_q, int32_t B, int32_t Hq,
                                     int32_t Hkv, int32_t T, float* out, void* workspace,
                                     size_t ws_bytes, void* stream) {
  if (!k_fp16) return fail(POT_ERR_INVALID_ARG, "k_fp16 is NULL");
  if (!aligned(k_fp16, 16)) return fail(POT_ERR_INVALID_ARG, "k_fp16 must be 16-byte aligned");
  DecodeArgs a{};
  a.q = q;
  a.k_f16 = k_fp16;
  a.v = v_cache;
  a.out = out;
  return decode_common(kScoreFp16, 0, a, kv_head_of_q, B, Hq, Hkv, T, t_cap, workspace, ws_bytes,
                       nullptr, stream);
}

}  // extern "C"
