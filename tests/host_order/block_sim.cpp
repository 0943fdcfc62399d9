// The norms around a block on the host (fibers.h): a call whose h is x and whose y is branch, or whose dx is dh and whose
// dbranch is dy, gives what the call with buffers of its own gives, whichever wave is ahead of the others.  Every
// combination of the two norms: where one is left out, so are the barriers of its sums.  Widths on both sides of every
// change of plan, the row's last vector cut at every place.
//
// block.hip is compiled as it stands, but for its launches (fibers::launch in the place of the triple brackets).
#include "fibers.h"

#include <string>

#include "block_host.inc"

// the compiler's function for the narrowing that the device has an instruction for
extern "C" __bf16 __truncsfbf2(float x) {
  uint32_t u = __float_as_uint(x);
  u += 0x7FFF + (u >> 16 & 1);
  return __builtin_bit_cast(__bf16, static_cast<uint16_t>(u >> 16));
}

namespace {

uint32_t random_state = 1;
float random_value() {  // in [-2, 2), a multiple of 2^-6, which bf16 holds
  random_state = random_state * 1664525u + 1013904223u;
  return static_cast<float>(random_state >> 24) / 64.0f - 2.0f;
}

struct Rows {
  std::vector<char> bytes;
  Rows(int64_t n, int32_t type, bool fill) : bytes(n * (type == EMB_BF16 ? 2 : 4)) {
    for (int64_t i = 0; fill && i < n; ++i) {
      const uint32_t u = __float_as_uint(random_value());
      if (type == EMB_BF16) {
        const uint16_t half = static_cast<uint16_t>(u >> 16);
        std::memcpy(&bytes[2 * i], &half, 2);
      } else {
        std::memcpy(&bytes[4 * i], &u, 4);
      }
    }
  }
  void* p() { return bytes.data(); }
};

long calls = 0;
bool check(const std::string& what, const Rows& a, const Rows& b) {
  ++calls;
  if (a.bytes == b.bytes) return true;
  size_t i = 0;
  while (a.bytes[i] == b.bytes[i]) ++i;
  std::printf("%s: in place other than with buffers of its own, from byte %zu of %zu\n", what.c_str(), i, a.bytes.size());
  return false;
}

bool run(int T, int D, int32_t st, int32_t bt, bool post, bool pre) {
  const std::string what = std::to_string(T) + " x " + std::to_string(D) + " types " + std::to_string(st) + " " +
                           std::to_string(bt) + (post ? " post" : "") + (pre ? " pre" : "");
  const int64_t n = static_cast<int64_t>(T) * D;
  const emb::DropMask none{0, nullptr, 0, 1.0f};
  const Rows x(n, st, true), branch(n, bt, true), dh(n, st, true), dy(n, bt, true);
  std::vector<float> post_stats(2 * T), pre_stats(2 * T), gate(D, 0.75f);
  bool ok = true;
  Rows h(n, st, false), y(n, bt, false), dx(n, st, false), db(n, bt, false);
  for (const bool in_place : {false, true})
    for (const bool last_first : {false, true}) {
      fibers::last_wave_first = last_first;
      Rows x2 = x, b2 = branch, h2(n, st, false), y2(n, bt, false);
      emb_block_norm_args f{};
      f.T = T, f.D = D, f.stream_dtype = st, f.dtype = bt;
      f.x = x2.p(), f.branch = b2.p(), f.gate = gate.data();
      f.h = in_place ? x2.p() : h2.p();
      f.y = !pre ? nullptr : in_place ? b2.p() : y2.p();
      f.ldx = f.ldb = f.ldh = f.ldy = D;
      f.alpha = 1.5, f.eps = 1e-5;
      f.post_stats = post ? post_stats.data() : nullptr;
      f.pre_stats = pre ? pre_stats.data() : nullptr;
      emb::launch_block_norm({&f, none}, nullptr);
      if (!in_place && !last_first) h = h2, y = y2;
      ok &= check("forward " + what + ", h", in_place ? x2 : h2, h);
      if (pre) ok &= check("forward " + what + ", y", in_place ? b2 : y2, y);
    }
  for (const bool in_place : {false, true})
    for (const bool last_first : {false, true}) {
      fibers::last_wave_first = last_first;
      Rows dh2 = dh, dy2 = dy, h2 = h, b2 = branch, dx2(n, st, false), db2(n, bt, false);
      emb_block_norm_grad_args g{};
      g.T = T, g.D = D, g.stream_dtype = st, g.dtype = bt;
      g.dh = dh2.p(), g.dy = pre ? dy2.p() : nullptr, g.h = h2.p(), g.branch = b2.p(), g.gate = gate.data();
      g.lddh = g.lddy = g.ldh = g.ldb = g.lddx = g.lddb = D;
      g.alpha = 1.5;
      g.post_stats = post ? post_stats.data() : nullptr;
      g.pre_stats = pre ? pre_stats.data() : nullptr;
      g.dx = in_place ? dh2.p() : dx2.p();
      g.dbranch = pre && in_place ? dy2.p() : db2.p();
      g.workspace_bytes = emb::block_norm_grad_workspace_bytes(T, D, 0);
      std::vector<char> workspace(g.workspace_bytes + 256);
      g.workspace = reinterpret_cast<void*>((reinterpret_cast<uintptr_t>(workspace.data()) + 255) & ~uintptr_t{255});
      emb::launch_block_norm_grad({&g, none}, nullptr);
      if (!in_place && !last_first) dx = dx2, db = db2;
      ok &= check("backward " + what + ", dx", in_place ? dh2 : dx2, dx);
      ok &= check("backward " + what + ", dbranch", pre && in_place ? dy2 : db2, db);
    }
  return ok;
}

}  // namespace

int main() {
  const int32_t types[3][2] = {{EMB_F32, EMB_F32}, {EMB_F32, EMB_BF16}, {EMB_BF16, EMB_BF16}};
  const int widths[] = {5, 61, 513, 1024, 1025, 1027, 1028, 1031, 1281, 1283, 1537, 1543, 2049, 2055, 3001, 4097, 8193};
  int bad = 0;
  for (const auto& t : types)
    for (const int D : widths)
      for (const int norms : {0, 1, 2, 3}) bad += !run(2, D, t[0], t[1], norms & 1, norms & 2);
  if (bad) return 1;
  std::printf("ok: %ld results, %ld stops of a lane\n", calls, fibers::stopped);
  return 0;
}
