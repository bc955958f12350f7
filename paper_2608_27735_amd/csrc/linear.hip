// linear.hip -- the linear layer: how a call becomes products (linear.h), copies of what
// 16-byte loads cannot take, and column sums.
#include <algorithm>

#include "linear_args.h"
#include "sides.h"

namespace abcd {
namespace {

#define LINEAR_BY_TYPE(l, fn, ...)                              \
  ((l).dtype == ABCD_F32   ? fn##_f32(__VA_ARGS__)              \
   : (l).dtype == ABCD_F16 ? fn##_f16(__VA_ARGS__)              \
                           : fn##_bf16(__VA_ARGS__))

// Whether the kernel for a few rows takes the forward: of up to 64, whose four products of 16 are
// made from one load of the weights, while the tiles' more even work does not pay for their second
// launch (bf16 with SiLU, weights from memory, by the bytes of weights for each 16 rows: 16 rows of
// 2,048 to 2,048, 8 MB, 5.6 against 9.6 us; 32 of 2,048 to 2,048, 16 MB, 8.8 against 10.0; 64 of 2,048
// to 2,048, 32 MB, 11.4 against 11.2; 64 of 2,048 to 4,096, 64 MB, 12.7 against 14.5; 32 of 4,096 to 4,096,
// 64 MB, 16.7 against 16.0; 64 of 4,096 to 2,560, 80 MB, 20.0 against 16.1; 32 of 8,192 to 8,192, 256
// MB, 55 against 33). Up to 16 always: they need no workspace (but 8,192 to 8,192 41 against 32).
bool few(const abcd_layer& l, int64_t n) {
  return n <= 16 || (n <= 64 && (n + 15) / 16 * l.o * l.i * (int64_t)type_bytes(l.dtype) <= 64 << 20);
}

// Room for the parts of the weights' gradient, none where the rows are too few to split: no
// more of them than run at once, and of a few tiles no more than their splits.
size_t dweight_part(const abcd_layer& l, int64_t steps) {
  const int64_t splits = dweight_splits(steps);
  if (splits == 1) return 0;
  auto room = [&](int64_t tile, int64_t slots) {
    return (size_t)std::min(slots, (l.o + tile - 1) / tile * ((l.i + tile - 1) / tile) * splits) * tile * tile;
  };
  return std::max(room(256, kBigSlots), room(128, kSmallSlots));
}

// Whether the narrow kernels do, in 16-bit types: wherever they hold the layer (bf16, SiLU,
// forward of 300,000 x 100 to 200 67 us, by the tiles 112, 1M x 130 to 20 101 against 324, 1,000 x 64
// to 64 9.8 against 11.0; backward of 20,000 x 64 to 64 18 against 31, 1,000 x 61 to 127 27.6 against
// 32.2), but forward not of long rows that are no whole vectors, whose weights take a load an
// element (300,000 x 200 to 100 80 against 71, 20,000 18 against 12).
bool narrow(const abcd_layer& l, int64_t n) {
  return l.dtype != ABCD_F32 && narrow_layer(l.i, l.o) && n > 64 &&
         (l.i <= 128 || l.o <= 64 || (l.i % 8 == 0 && l.o % 8 == 0));
}
bool narrow_bwd(const abcd_layer& l, int64_t n) { return l.dtype != ABCD_F32 && narrow_layer_bwd(l.i, l.o) && n > 0; }
int64_t narrow_blocks(int64_t n) { return std::min<int64_t>((n + 127) / 128, 4 * kCUs); }
int64_t narrow_bwd_blocks(int64_t n) { return std::min<int64_t>((n + 127) / 128, 2 * kCUs); }

struct Scratch {
  void *x, *w, *dz;
  float *part, *sums;
  size_t bytes;
};

Scratch layout(const abcd_layer& l, int64_t n, bool backward, void* workspace) {
  const size_t sz = type_bytes(l.dtype);
  const int64_t step = kStepBytes / (int64_t)sz;
  auto steps = [&](int64_t kn) { return (kn + step - 1) / step; };
  Pieces p{static_cast<char*>(workspace)};
  Scratch s{};
  if (!backward && (few(l, n) || narrow(l, n))) return s;
  if (backward && narrow_bwd(l, n)) {
    s.part = static_cast<float*>(p.take(narrow_bwd_blocks(n) * (l.o * l.i + l.o) * sizeof(float)));
    s.bytes = p.used;
    return s;
  }
  s.x = p.take(n * up8(l.i) * sz);
  s.w = p.take(l.o * up8(l.i) * sz);
  size_t part = product_part(sz, n, l.o, 1, steps(l.i));
  if (backward) {
    s.dz = p.take(n * up8(l.o) * sz);
    part = std::max({part, product_part(sz, n, l.i, 1, steps(l.o)), (size_t)(sum_parts_of(n) * l.o),
                     dweight_part(l, steps(n))});
    s.sums = static_cast<float*>(p.take(std::max(sum_parts_of(n), few(l, n) ? few_parts(n) : 0) * l.o * sizeof(float)));
  }
  s.part = static_cast<float*>(p.take(part * sizeof(float)));
  s.bytes = p.used;
  return s;
}

}  // namespace

size_t linear_workspace_bytes(const abcd_layer& l, int64_t n, bool backward) {
  return layout(l, n, backward, nullptr).bytes;
}

int32_t launch_linear(const abcd_layer& l, int64_t n, const void* x, int64_t ldx, const void* residual, int64_t ldr,
                      void* y, int64_t ldy, void* slope, void* workspace, hipStream_t stream) {
  if (n == 0) return ABCD_OK;
  const Scratch s = layout(l, n, false, workspace);
  LinearOut out{Side{{x, nullptr}, ldx, n}, Side{{l.w, nullptr}, l.i, l.o}, l.b, residual, y,
                l.act == ABCD_ACT_NONE ? nullptr : slope, l.i, l.o, ldr, ldy, up8(l.o), l.act, Tiling{s.part, 0, 0, 1, 0}};
  if (narrow(l, n)) {
    const LinearNarrow a{x, l.w, l.b, residual, y, out.slope, n, l.i, l.o, ldx, ldr, ldy, out.ldslope, l.act};
    return l.dtype == ABCD_F16 ? linear_narrow_f16(a, narrow_blocks(n), stream) : linear_narrow_bf16(a, narrow_blocks(n), stream);
  }
  if (few(l, n)) return LINEAR_BY_TYPE(l, linear_few, out, stream);
  Packs copies;
  out.x = side_of(copies, l.dtype, x, n, l.i, ldx, s.x);
  out.w = side_of(copies, l.dtype, l.w, l.o, l.i, l.i, s.w);
  TRY_STATUS(launch(copies, l.dtype, stream));
  return LINEAR_BY_TYPE(l, linear_out, out, stream);
}

int32_t launch_linear_bwd(const abcd_layer& l, int64_t n, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                          const int8_t* q, const uint8_t* e, const void* slope, void* dx, int64_t lddx, void* dw, void* db,
                          void* workspace, hipStream_t stream) {
  const Scratch s = layout(l, n, true, workspace);
  if (l.act == ABCD_ACT_NONE) slope = nullptr;
  if (narrow_bwd(l, n)) {
    const LinearNarrowBwd a{x, q, e, dy, slope, l.w, l.b, dx, dw || db ? s.part : nullptr, n, l.i, l.o, ldx, lddy, up8(l.o),
                            lddx, l.act};
    const int64_t blocks = narrow_bwd_blocks(n);
    TRY_STATUS(l.dtype == ABCD_F16 ? linear_narrow_bwd_f16(a, blocks, stream) : linear_narrow_bwd_bf16(a, blocks, stream));
    if (!a.part) return ABCD_OK;
    SumOuts outs{};
    outs.add(dw, l.o * l.i);
    outs.add(db, l.o);
    return launch_sum_parts(s.part, blocks, outs, l.dtype, stream);
  }
  const bool again = l.act != ABCD_ACT_NONE && !slope;
  auto sum_up = [&](int64_t parts) -> int32_t {
    SumOuts outs{};
    outs.add(db, l.o);
    return launch_sum_parts(s.sums, parts, outs, l.dtype, stream);
  };
  const bool one = sum_parts_of(n) == 1;  // part of the bias's sums, which is then all of them
  const int lanes = std::min(lanes_for((int)(up8(l.o) / 8)), 64);
  Side xs{}, w{}, dz{};
  if (n > 0) {
    Packs copies;
    const bool tiles = again && !few(l, n);
    if (again || dw) {
      if (q) {
        // a checkpoint's rows up to a multiple of 8: zeros behind their end
        TRY_STATUS(launch_unpack8(l.dtype, n, up8(l.i), q, e, s.x, up8(l.i), stream));
        xs = Side{{s.x, nullptr}, up8(l.i), n};
      } else if (tiles || dw) {
        xs = side_of(copies, l.dtype, x, n, l.i, ldx, s.x);
      }
    }
    if (tiles || dx) w = side_of(copies, l.dtype, l.w, l.o, l.i, l.i, s.w);
    if (l.act == ABCD_ACT_NONE)
      dz = side_of(copies, l.dtype, dy, n, l.o, lddy, s.dz);
    else
      dz = Side{{s.dz, nullptr}, up8(l.o), n};
    TRY_STATUS(launch(copies, l.dtype, stream));
    if (again && !tiles) {
      // the weights as they lie in memory, and x: a checkpoint's copy or the rows themselves
      LinearOut a{q ? xs : Side{{x, nullptr}, ldx, n}, Side{{l.w, nullptr}, l.i, l.o}, l.b, nullptr, s.dz, nullptr, l.i, l.o,
                  0, dz.ld, 0, l.act, Tiling{}};
      a.dy = dy;
      a.lddy = lddy;
      if (db && few_parts(n) == 1)
        a.db = db;
      else if (db)
        a.part = s.sums;
      TRY_STATUS(LINEAR_BY_TYPE(l, linear_few, a, stream));
    } else if (again) {
      const LinearDz a{xs, w, l.b, dy, s.dz, l.i, l.o, lddy, dz.ld, l.act, Tiling{s.part, 0, 0, 1, 0}};
      TRY_STATUS(LINEAR_BY_TYPE(l, linear_dz, a, stream));
    } else if (slope) {
      const LinearSlope a{dy, slope, s.dz, db && !one ? s.sums : nullptr, one ? db : nullptr, n, l.o, lddy, up8(l.o), dz.ld, lanes};
      TRY_STATUS(LINEAR_BY_TYPE(l, linear_slope, a, sum_parts_of(n), stream));
    }
    if (dx) {
      // W across: its index is i, the contraction o
      const LinearDx a{dz, Side{{w.p[0], nullptr}, w.ld, l.i}, dx, l.o, l.i, lddx, Tiling{s.part, 0, 0, 1, 0}};
      TRY_STATUS(LINEAR_BY_TYPE(l, linear_dx, a, stream));
    }
  }
  if (dw) {
    FfnDWeight a{};
    a.part = s.part;
    a.n = n;
    a.one[a.count++] = FfnDWeight::One{dz.p[0], xs.p[0], dw, dz.ld, l.o, xs.ld, l.i, 1.0f, 0, 0, 0};
    TRY_STATUS(LINEAR_BY_TYPE(l, linear_dw, a, stream));
  }
  if (!db) return ABCD_OK;
  if (n > 0 && again && few(l, n)) return few_parts(n) == 1 ? ABCD_OK : sum_up(few_parts(n));
  if (n > 0 && slope) return one ? ABCD_OK : sum_up(sum_parts_of(n));
  if (n > 0 && one) {
    const LinearSlope a{dz.p[0], nullptr, nullptr, nullptr, db, n, l.o, dz.ld, 0, up8(l.o), lanes};
    return LINEAR_BY_TYPE(l, linear_slope, a, 1, stream);
  }
  SumCall sums{l.dtype, n, s.part};
  sums.add(db, dz.p[0], dz.ld, l.o, 1.0f);
  return sums.launch(stream);
}

}  // namespace abcd
