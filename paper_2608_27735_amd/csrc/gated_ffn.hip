// gated_ffn.hip -- the gated feed-forward block: how a call becomes products
// (gated_ffn.h), copies of what 16-byte loads cannot take, and column sums.
#include <algorithm>

#include "sides.h"

namespace abcd {
namespace {

struct Scratch {
  void *x, *wg, *wu, *wd, *dz, *gate, *up, *hidden;
  float *part, *dx_part;
  size_t bytes;
};

// Room for the parts of the weights' gradients, none where the rows are too few to
// split: no more of them than run at once, and of a few tiles no more than their splits.
size_t dweight_part(const abcd_ffn& f, int64_t steps) {
  const int64_t splits = dweight_splits(steps);
  if (splits == 1) return 0;
  auto room = [&](int64_t tile, int64_t slots) {
    auto of = [&](int64_t rows, int64_t cols) { return (rows + tile - 1) / tile * ((cols + tile - 1) / tile); };
    return (size_t)std::min(slots, (2 * of(f.h, f.d) + of(f.o, f.h)) * splits) * tile * tile;
  };
  return std::max(room(256, kBigSlots), room(128, kSmallSlots));
}

// Whether the kernels for a few rows take the first products. They read x again for
// every 16 columns of h, so that many rows of a wide block leave it to the tiles: bf16,
// 64 x 512 x 1,376 x 512 16 against 19 us, 64 x 1,024 x 2,816 x 1,024 24 either way, 64 x
// 2,048 x 5,632 x 2,048 52 against 35; fp32, 32 rows of the second 30 against 37, 48 rows
// 41 against 38.
bool few(const abcd_ffn& f, int64_t n) {
  return n <= 16 || (n <= 64 && (n + 15) / 16 * (2 * f.h * f.d + f.o * f.h) * (int64_t)type_bytes(f.dtype) <= 80 << 20);
}
// Whether the narrow kernels do, in 16-bit types, of what they hold in registers and LDS.
// Both ways they win from the first row on, with fewer launches (64 x 128 x 64, forward
// and backward: one row 49 against 68 us, 100 rows 48 against 73, 16,000 42 against 60; of 384 hidden units,
// 8,000 rows lose, 94 against 80, and 32,000 win, 103 against 120). The forwards of the
// larger shapes have their setting up to make good: 128 x 192 x 128, 32,000 rows 22
// against 20 us, 64,000 25 against 32.
bool narrow_forward(const abcd_ffn& f, int64_t n) {
  const int shape = f.dtype == ABCD_F32 ? 0 : narrow_shape(f.d, f.h, f.o);
  return shape > 0 && (shape <= 2 || n >= 40000);
}
bool narrow(const abcd_ffn& f, int64_t n) { return narrow_forward(f, n) && narrow_shape(f.d, f.h, f.o) <= 2; }
int64_t narrow_blocks(const abcd_ffn& f, int64_t n) {
  return std::min<int64_t>((n + 255) / 256, (narrow_shape(f.d, f.h, f.o) == 1 ? 2 : 1) * kCUs);
}
int64_t narrow_bwd_blocks(int64_t n) { return std::min<int64_t>((n + 63) / 64, kCUs); }
int64_t narrow_sums(const abcd_ffn& f) { return 2 * f.h * f.d + f.o * f.h + 2 * f.h + f.o; }

Scratch layout(const abcd_ffn& f, int64_t n, bool saved, bool backward, void* workspace) {
  const size_t sz = type_bytes(f.dtype);
  const int64_t dp = up8(f.d), hp = up8(f.h), op = up8(f.o);
  Pieces p{static_cast<char*>(workspace)};
  Scratch s{};
  if (!saved && (backward ? narrow(f, n) : narrow_forward(f, n))) {
    if (backward) {
      s.part = static_cast<float*>(p.take(narrow_bwd_blocks(n) * narrow_groups(f.h) * narrow_sums(f) * sizeof(float)));
      if (f.h > 128) s.dx_part = static_cast<float*>(p.take(n * up8(f.d) * sizeof(float)));
    }
    s.bytes = p.used;
    return s;
  }
  if (!backward && few(f, n)) {
    if (!saved) s.hidden = p.take(n * hp * sz);
    s.bytes = p.used;
    return s;
  }
  s.x = p.take(n * dp * sz);
  s.wg = p.take(f.h * dp * sz);
  s.wu = p.take(f.h * dp * sz);
  s.wd = p.take(f.o * hp * sz);
  if (!saved) s.hidden = p.take(n * hp * sz);
  const int64_t step = kStepBytes / (int64_t)sz;
  auto steps = [&](int64_t kn) { return (kn + step - 1) / step; };
  size_t part = 0;
  if (!backward || !saved) part = product_part(sz, n, f.h, 2, steps(f.d));
  if (!backward) part = std::max(part, product_part(sz, n, f.o, 1, steps(f.h)));
  if (backward) {
    s.dz = p.take(n * op * sz);
    s.gate = p.take(n * hp * sz);
    s.up = p.take(n * hp * sz);
    part = std::max({part, product_part(sz, n, f.h, 1, steps(f.o)), product_part(sz, n, f.d, 1, 2 * steps(f.h)),
                     (size_t)sum_parts_of(n) * (2 * f.h + f.o), dweight_part(f, steps(n))});
  }
  s.part = static_cast<float*>(p.take(part * sizeof(float)));
  s.bytes = p.used;
  return s;
}

#define FFN_BY_TYPE(f, fn, ...)                                 \
  ((f).dtype == ABCD_F32   ? fn##_f32(__VA_ARGS__)              \
   : (f).dtype == ABCD_F16 ? fn##_f16(__VA_ARGS__)              \
                           : fn##_bf16(__VA_ARGS__))

// Both projections as one side of two halves; their copies are laid out alike.
Side gate_up(Packs& p, const abcd_ffn& f, const Scratch& s) {
  if (direct(f.dtype, f.w_gate, f.d, f.d) && direct(f.dtype, f.w_up, f.d, f.d))
    return Side{{f.w_gate, f.w_up}, f.d, f.h};
  add_pack(p, f.dtype, f.h, f.d, f.w_gate, f.d, s.wg, up8(f.d), DropKey{});
  add_pack(p, f.dtype, f.h, f.d, f.w_up, f.d, s.wu, up8(f.d), DropKey{});
  return Side{{s.wg, s.wu}, up8(f.d), f.h};
}

int32_t few_in(const abcd_ffn& f, int64_t n, const void* x, int64_t ldx, void* by_gate, void* by_up, void* hidden,
               hipStream_t stream) {
  const FfnIn in{Side{{x, nullptr}, ldx, n}, Side{{f.w_gate, f.w_up}, f.d, f.h}, f.b_gate, f.b_up, hidden, by_gate,
                 by_up, f.d, f.h, up8(f.h), f.act, Tiling{}};
  return FFN_BY_TYPE(f, ffn_few_in, in, stream);
}

}  // namespace

bool gated_ffn_keeps(const abcd_ffn& f, int64_t n) { return !narrow(f, n); }

// Never 0, also of a call that needs none: which those are is not the caller's to know.
size_t gated_ffn_workspace_bytes(const abcd_ffn& f, int64_t n, bool saved, bool backward) {
  return std::max<size_t>(256, layout(f, n, saved, backward, nullptr).bytes);
}

int32_t launch_gated_ffn(const abcd_ffn& f, int64_t n, const void* x, int64_t ldx, const void* residual,
                         int64_t ldr, void* y, int64_t ldy, void* by_gate, void* by_up, void* hidden, void* workspace,
                         hipStream_t stream) {
  if (n == 0) return ABCD_OK;
  if (!hidden && narrow_forward(f, n)) {
    const FfnNarrow a{x, f.w_gate, f.w_up, f.w_down, f.b_gate, f.b_up, f.b_down, residual, y, n, f.d, f.h, f.o,
                      ldx, ldr, ldy, drop_key(f.p, f.seed, f.offset), f.act};
    return f.dtype == ABCD_F16 ? ffn_narrow_f16(a, narrow_blocks(f, n), stream)
                               : ffn_narrow_bf16(a, narrow_blocks(f, n), stream);
  }
  const Scratch s = layout(f, n, hidden != nullptr, false, workspace);
  if (!hidden) hidden = s.hidden;
  const int64_t hp = up8(f.h);
  FfnOut out{Side{{hidden, nullptr}, hp, n}, Side{{f.w_down, nullptr}, f.h, f.o}, f.b_down, residual, y, f.h, f.o, ldr,
             ldy, drop_key(f.p, f.seed, f.offset), Tiling{s.part, 0, 0, 1, 0}};
  if (few(f, n)) {
    TRY_STATUS(few_in(f, n, x, ldx, by_gate, by_up, hidden, stream));
    return FFN_BY_TYPE(f, ffn_few_out, out, stream);
  }
  Packs copies;
  const Side xs = side_of(copies, f.dtype, x, n, f.d, ldx, s.x), w = gate_up(copies, f, s);
  out.w = side_of(copies, f.dtype, f.w_down, f.o, f.h, f.h, s.wd);
  TRY_STATUS(launch(copies, f.dtype, stream));
  const FfnIn in{xs, w, f.b_gate, f.b_up, hidden, by_gate, by_up, f.d, f.h, hp, f.act, Tiling{s.part, 0, 0, 1, 0}};
  TRY_STATUS(FFN_BY_TYPE(f, ffn_in, in, stream));
  return FFN_BY_TYPE(f, ffn_out, out, stream);
}

int32_t launch_gated_ffn_bwd(const abcd_ffn& f, int64_t n, const void* dy, int64_t lddy, const void* x,
                             int64_t ldx, const void* by_gate, const void* by_up, const void* hidden, void* dx,
                             int64_t lddx, void* dw_gate, void* dw_up, void* dw_down, void* db_gate, void* db_up,
                             void* db_down, void* workspace, hipStream_t stream) {
  const Scratch s = layout(f, n, hidden != nullptr, true, workspace);
  const int64_t hp = up8(f.h);
  // dz is dy with zeros where the forward dropped; the factor of what is kept
  // multiplies the sums that dz enters
  DropKey mask = drop_key(f.p, f.seed, f.offset);
  const float scale = mask.scale;
  mask.scale = 1.0f;
  if (!hidden && narrow(f, n)) {
    const int64_t blocks = narrow_bwd_blocks(n);
    const int64_t sz = (int64_t)type_bytes(f.dtype);
    auto from = [&](const void* p, int64_t e) { return p ? static_cast<const char*>(p) + e * sz : nullptr; };
    // no rows: no parts either, whose sums are zeros
    for (int64_t c = 0; n > 0 && c < f.h; c += 128) {
      const FfnNarrowBwd a{x, dy, from(f.w_gate, c * f.d), from(f.w_up, c * f.d), from(f.w_down, c), from(f.b_gate, c),
                           from(f.b_up, c), dx, s.part, s.dx_part, n, f.d, std::min<int64_t>(f.h - c, 128), f.o, f.h,
                           c, ldx, lddy, lddx, up8(f.d), narrow_sums(f), c + 128 >= f.h, mask, scale, f.act};
      TRY_STATUS(f.dtype == ABCD_F16 ? ffn_narrow_bwd_f16(a, blocks, stream) : ffn_narrow_bwd_bf16(a, blocks, stream));
    }
    SumOuts outs{};
    outs.add(dw_gate, f.h * f.d);
    outs.add(dw_up, f.h * f.d);
    outs.add(dw_down, f.o * f.h);
    outs.add(db_gate, f.h);
    outs.add(db_up, f.h);
    outs.add(db_down, f.o);
    return launch_sum_parts(s.part, blocks * narrow_groups(f.h), outs, f.dtype, stream);
  }
  Side xs{}, wgu{}, wd{}, dz{};
  if (n > 0) {
    Packs copies;
    xs = side_of(copies, f.dtype, x, n, f.d, ldx, s.x);
    wgu = gate_up(copies, f, s);
    wd = side_of(copies, f.dtype, f.w_down, f.o, f.h, f.h, s.wd);
    if (f.p > 0.0) {
      dz = Side{{s.dz, nullptr}, up8(f.o), n};
      add_pack(copies, f.dtype, n, f.o, dy, lddy, s.dz, dz.ld, mask);
    } else {
      dz = side_of(copies, f.dtype, dy, n, f.o, lddy, s.dz);
    }
    TRY_STATUS(launch(copies, f.dtype, stream));
    if (!hidden && few(f, n)) {
      TRY_STATUS(few_in(f, n, x, ldx, s.gate, s.up, s.hidden, stream));
      by_gate = s.gate;
      by_up = s.up;
      hidden = s.hidden;
    } else if (!hidden) {
      const FfnIn in{xs, wgu, f.b_gate, f.b_up, s.hidden, s.gate, s.up, f.d, f.h, hp, f.act, Tiling{s.part, 0, 0, 1, 0}};
      TRY_STATUS(FFN_BY_TYPE(f, ffn_in, in, stream));
      by_gate = s.gate;
      by_up = s.up;
      hidden = s.hidden;
    }
  }
  // W side across: its index is h, the contraction o
  const bool inner = dx || dw_gate || dw_up || db_gate || db_up;
  if (n > 0 && inner) {
    const FfnDHidden dh{dz, Side{{wd.p[0], nullptr}, wd.ld, f.h}, by_gate, by_up, s.gate, s.up, f.o, f.h, hp, scale, Tiling{s.part, 0, 0, 1, 0}};
    TRY_STATUS(FFN_BY_TYPE(f, ffn_dhidden, dh, stream));
  }
  const Side dgu{{s.gate, s.up}, hp, n};
  if (n > 0 && dx) {
    const FfnDX a{dgu, Side{{wgu.p[0], wgu.p[1]}, wgu.ld, f.d}, dx, f.h, f.d, lddx, Tiling{s.part, 0, 0, 1, 0}};
    TRY_STATUS(FFN_BY_TYPE(f, ffn_dx, a, stream));
  }
  FfnDWeight dw{};
  dw.part = s.part;
  dw.n = n;
  auto want = [&](void* out, const void* m, int64_t ld, int64_t rows, const Side& w, int64_t cols, float factor) {
    if (out) dw.one[dw.count++] = FfnDWeight::One{m, w.p[0], out, ld, rows, w.ld, cols, factor, 0, 0, 0};
  };
  want(dw_gate, s.gate, hp, f.h, xs, f.d, 1.0f);
  want(dw_up, s.up, hp, f.h, xs, f.d, 1.0f);
  want(dw_down, dz.p[0], dz.ld, f.o, Side{{hidden, nullptr}, hp, 0}, f.h, scale);
  if (dw.count > 0) TRY_STATUS(FFN_BY_TYPE(f, ffn_dweight, dw, stream));
  SumCall sums{f.dtype, n, s.part};
  sums.add(db_gate, s.gate, hp, f.h, 1.0f);
  sums.add(db_up, s.up, hp, f.h, 1.0f);
  sums.add(db_down, dz.p[0], dz.ld, f.o, scale);
  return sums.launch(stream);
}

}  // namespace abcd
