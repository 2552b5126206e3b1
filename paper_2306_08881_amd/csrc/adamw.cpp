// C ABI of the AdamW operators: state binding, gradient slots, argument checks and launches.  Every
// check runs on the host before anything is enqueued.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <string>
#include <vector>

#include "acp.h"
#include "adamw_internal.hpp"

namespace acp {
hipError_t adamw_launch_step(const AwSlotPlan& s, int bits, const AwArgs& a, hipStream_t st);
hipError_t adamw_launch_norm(const AwSlotPlan& s, AwNormArgs a, hipStream_t st);
}  // namespace acp

namespace {

struct Span {
  uintptr_t first, last;
  bool write;
};

}  // namespace

struct acp_adamw {
  acp::AwPlan plan;
  uint8_t* dev = nullptr;   // bound state block
  int device = -1;
  bool has_params = false;
  struct Slot {
    acp::AwSlotPlan plan;
    uint8_t* dev = nullptr;  // the slot's gradient block
  };
  Slot slots[acp::kAwSlots];
  // what the calls write (state, parameters, copies, the slots' blocks) and what they read (the slots'
  // gradients), each sorted and without overlaps
  std::vector<Span> written, read;
  mutable std::string err;
};

namespace {

acp_status fail(const acp_adamw* o, acp_status s, const std::string& msg) {
  if (o) o->err = msg;
  return s;
}
// The same of a fixed text, also when the host has no memory for it (the last error then stays).
acp_status fail(const acp_adamw* o, acp_status s, const char* msg) noexcept {
  try {
    if (o) o->err = msg;
  } catch (...) {
  }
  return s;
}

// No C++ exception leaves a C entry: what is left to throw is the host's memory running out.
template <class F>
acp_status guarded(const acp_adamw* o, F f) {
  try {
    return f();
  } catch (...) {
    return fail(o, ACP_E_STATE, "out of host memory");
  }
}

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

acp_status check_device(const acp_adamw* o) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return fail(o, ACP_E_DEVICE, "hipGetDevice failed");
  if (dev != o->device) return fail(o, ACP_E_INVALID, "the device current at bind time must be current for this call");
  return ACP_OK;
}

// Whether any two spans meet of which one at least is written.
bool clash(std::vector<Span>& v) {
  std::sort(v.begin(), v.end(), [](const Span& x, const Span& y) { return x.first < y.first; });
  uintptr_t any = 0, written = 0;  // ends of what came before
  for (const Span& s : v) {
    if (s.first < written || (s.write && s.first < any)) return true;
    any = std::max(any, s.last);
    if (s.write) written = std::max(written, s.last);
  }
  return false;
}

void add(std::vector<Span>& v, const void* p, int64_t bytes, bool write) {
  if (!p || bytes <= 0) return;
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  v.push_back(Span{a, a + static_cast<uintptr_t>(bytes), write});
}

// the spans of the bound state and parameters
void state_spans(const acp_adamw* o, std::vector<Span>& v) {
  add(v, o->dev, o->plan.total_bytes, true);
  for (const acp::AwTensor& t : o->plan.tensors) {
    add(v, t.p, t.n * t.m * 4, true);
    add(v, t.copy, t.n * t.m * 2, true);
  }
}

// the spans of a slot's block and gradients
void slot_spans(const acp_adamw* o, const acp::AwSlotPlan& s, const void* block, std::vector<Span>& v) {
  add(v, block, s.total_bytes, true);
  for (size_t i = 0; i < s.grads.size(); ++i) {
    const acp::AwGrad& g = s.grads[i];
    const acp::AwTensor& t = o->plan.tensors[i];
    add(v, g.g, t.n * t.m * (g.bf16 ? 2 : 4), false);
    add(v, g.a, t.n * g.rank * 4, false);
    add(v, g.b, t.m * g.rank * 4, false);
  }
}

// Those spans that are written, or only read, with overlapping and adjoining ones as one (v is sorted).
std::vector<Span> merged(const std::vector<Span>& v, bool write) {
  std::vector<Span> out;
  for (const Span& s : v) {
    if (s.write != write) continue;
    if (!out.empty() && s.first <= out.back().last)
      out.back().last = std::max(out.back().last, s.last);
    else
      out.push_back(s);
  }
  return out;
}

// Whether `bytes` from p on meet any of the spans (of merged()).
bool meets(const std::vector<Span>& v, const void* p, int64_t bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  const auto next = std::upper_bound(v.begin(), v.end(), a, [](uintptr_t x, const Span& s) { return x < s.first; });
  return (next != v.end() && next->first < a + static_cast<uintptr_t>(bytes)) || (next != v.begin() && a < (next - 1)->last);
}

// the gradients' values and factors
acp_status take_grads(const acp_adamw* o, const acp_adamw_grad* grads, acp::AwSlotPlan& s) {
  if (!grads) return fail(o, ACP_E_INVALID, "grads is NULL");
  for (size_t i = 0; i < o->plan.tensors.size(); ++i) {
    const acp_adamw_grad& x = grads[i];
    const acp::AwTensor& t = o->plan.tensors[i];
    const std::string at = " (tensor " + std::to_string(i) + ")";
    acp::AwGrad g{};
    if (x.rank < 0 || x.rank > acp::kAwMaxRank) return fail(o, ACP_E_INVALID, "rank out of range" + at);
    if (x.type != ACP_GRAD_FP32 && x.type != ACP_GRAD_BF16) return fail(o, ACP_E_INVALID, "unknown gradient type" + at);
    if (x.rank > 0) {
      if (!x.a || !x.b) return fail(o, ACP_E_INVALID, "null factor" + at);
      if (x.type != ACP_GRAD_FP32) return fail(o, ACP_E_UNSUPPORTED, "factors are fp32" + at);
      if (!aligned(x.a, 4) || !aligned(x.b, 4)) return fail(o, ACP_E_INVALID, "misaligned factor" + at);
      if (t.n > acp::kAwMaxFactorRows || t.m > acp::kAwMaxFactorCols) return fail(o, ACP_E_UNSUPPORTED, "too large for factors" + at);
      g.a = x.a;
      g.b = x.b;
      g.rank = x.rank;
    } else {
      if (!x.grad) return fail(o, ACP_E_INVALID, "null gradient" + at);
      if (!aligned(x.grad, x.type == ACP_GRAD_FP32 ? 4 : 2)) return fail(o, ACP_E_INVALID, "misaligned gradient" + at);
      g.g = x.grad;
      g.bf16 = x.type == ACP_GRAD_BF16;
    }
    s.grads.push_back(g);
  }
  const std::string msg = acp::adamw_slot(s, o->plan);
  return msg.empty() ? ACP_OK : fail(o, ACP_E_INVALID, msg);
}

acp_status check_slot(const acp_adamw* o, int32_t slot) {
  if (slot < 0 || slot >= acp::kAwSlots) return fail(o, ACP_E_INVALID, "gradient slot out of range");
  if (!o->dev) return fail(o, ACP_E_STATE, "state not bound");
  if (!o->slots[slot].dev) return fail(o, ACP_E_STATE, "no gradients in this slot");
  return check_device(o);
}

}  // namespace

extern "C" {

acp_status acp_adamw_init(acp_adamw** out, int32_t num_tensors, const int32_t* ndims, const int64_t* dims,
                          int32_t moment_bits, const uint8_t* no_decay, uint64_t seed) {
  if (!out) return ACP_E_INVALID;
  *out = nullptr;
  return guarded(nullptr, [&]() -> acp_status {
    acp::AwPlan plan;
    if (!acp::adamw_plan(plan, num_tensors, ndims, dims, moment_bits, no_decay, seed).empty()) return ACP_E_INVALID;
    acp_adamw* o = new acp_adamw();
    o->plan = std::move(plan);
    *out = o;
    return ACP_OK;
  });
}

acp_status acp_adamw_state_bytes(const acp_adamw* o, int64_t* bytes) {
  if (!o || !bytes) return fail(o, ACP_E_INVALID, "null argument");
  *bytes = o->plan.total_bytes;
  return ACP_OK;
}

acp_status acp_adamw_bind(acp_adamw* o, void* device_ptr, int64_t bytes, float* const* params,
                          uint16_t* const* copies, void* stream) {
  if (!o) return ACP_E_INVALID;
  return guarded(o, [&]() -> acp_status {
    if (!device_ptr) return fail(o, ACP_E_INVALID, "device_ptr is NULL");
    if (!aligned(device_ptr, 256)) return fail(o, ACP_E_INVALID, "state block must be 256-byte aligned");
    if (bytes < o->plan.total_bytes) return fail(o, ACP_E_STATE, "state block too small");
    if (copies && !params) return fail(o, ACP_E_INVALID, "copies without parameters");
    std::vector<acp::AwTensor> ts = o->plan.tensors;
    std::vector<Span> spans;
    add(spans, device_ptr, o->plan.total_bytes, true);
    for (size_t i = 0; i < ts.size(); ++i) {
      ts[i].p = params ? params[i] : nullptr;
      ts[i].copy = copies ? copies[i] : nullptr;
      if (params && !params[i]) return fail(o, ACP_E_INVALID, "null parameter");
      if (!aligned(ts[i].p, 4) || !aligned(ts[i].copy, 2)) return fail(o, ACP_E_INVALID, "misaligned parameter");
      add(spans, ts[i].p, ts[i].n * ts[i].m * 4, true);
      add(spans, ts[i].copy, ts[i].n * ts[i].m * 2, true);
    }
    if (clash(spans)) return fail(o, ACP_E_INVALID, "parameters, copies and the state block overlap");
    std::vector<Span> written = merged(spans, true);
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return fail(o, ACP_E_DEVICE, "hipGetDevice failed");
    hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t* d = static_cast<uint8_t*>(device_ptr);
    o->dev = nullptr;
    for (auto& x : o->slots) x = acp_adamw::Slot{};
    hipError_t e = hipMemsetAsync(d, 0, o->plan.off_tensors, s);
    if (e == hipSuccess)
      e = hipMemcpyAsync(d + o->plan.off_tensors, ts.data(), ts.size() * sizeof(acp::AwTensor), hipMemcpyHostToDevice, s);
    if (e == hipSuccess) e = hipStreamSynchronize(s);
    if (e != hipSuccess) return fail(o, ACP_E_DEVICE, std::string("bind failed: ") + hipGetErrorString(e));
    o->plan.tensors.swap(ts);
    o->written.swap(written);
    o->read.clear();
    o->dev = d;
    o->device = dev;
    o->has_params = params != nullptr;
    o->err.clear();
    return ACP_OK;
  });
}

acp_status acp_adamw_regions(const acp_adamw* o, int64_t* elems, int64_t* blocks, int64_t* m_off, int64_t* v_off,
                             int64_t* m_scale_off, int64_t* v_scale_off) {
  if (!o) return ACP_E_INVALID;
  if (elems) *elems = o->plan.elems;
  if (blocks) *blocks = o->plan.bits == 8 ? o->plan.blocks : 0;
  if (m_off) *m_off = o->plan.off_m;
  if (v_off) *v_off = o->plan.off_v;
  if (m_scale_off) *m_scale_off = o->plan.off_ms;
  if (v_scale_off) *v_scale_off = o->plan.off_vs;
  return ACP_OK;
}

acp_status acp_adamw_tensor_info(const acp_adamw* o, int32_t tensor, int64_t* first, int64_t* first_block,
                                 int64_t* blocks, int32_t* block_rows, int32_t* block_cols) {
  if (!o) return ACP_E_INVALID;
  if (tensor < 0 || tensor >= static_cast<int32_t>(o->plan.tensors.size()))
    return fail(o, ACP_E_INVALID, "tensor out of range");
  const acp::AwTensor& t = o->plan.tensors[tensor];
  if (first) *first = t.off;
  if (first_block) *first_block = t.blk;
  if (blocks) *blocks = t.blocks;
  if (block_rows) *block_rows = t.k;
  if (block_cols) *block_cols = t.w / t.k;
  return ACP_OK;
}

acp_status acp_adamw_grads_bytes(const acp_adamw* o, const acp_adamw_grad* grads, int64_t* bytes) {
  if (!o || !bytes) return fail(o, ACP_E_INVALID, "null argument");
  return guarded(o, [&]() -> acp_status {
    acp::AwSlotPlan s;
    const acp_status st = take_grads(o, grads, s);
    if (st == ACP_OK) *bytes = s.total_bytes;
    return st;
  });
}

acp_status acp_adamw_set_grads(acp_adamw* o, int32_t slot, const acp_adamw_grad* grads, void* device_ptr,
                               int64_t bytes, void* stream) {
  if (!o) return ACP_E_INVALID;
  return guarded(o, [&]() -> acp_status {
    if (slot < 0 || slot >= acp::kAwSlots) return fail(o, ACP_E_INVALID, "gradient slot out of range");
    if (!o->dev) return fail(o, ACP_E_STATE, "state not bound");
    if (!device_ptr) return fail(o, ACP_E_INVALID, "device_ptr is NULL");
    if (!aligned(device_ptr, 256)) return fail(o, ACP_E_INVALID, "gradient block must be 256-byte aligned");
    acp::AwSlotPlan s;
    acp_status st = take_grads(o, grads, s);
    if (st != ACP_OK) return st;
    if (bytes < s.total_bytes) return fail(o, ACP_E_STATE, "gradient block too small");
    std::vector<Span> spans;
    state_spans(o, spans);
    slot_spans(o, s, device_ptr, spans);
    for (int32_t i = 0; i < acp::kAwSlots; ++i)
      if (i != slot && o->slots[i].dev) slot_spans(o, o->slots[i].plan, o->slots[i].dev, spans);
    if (clash(spans))
      return fail(o, ACP_E_INVALID, "gradients or the gradient block overlap the parameters, the state or another slot's");
    std::vector<Span> written = merged(spans, true), read = merged(spans, false);
    if ((st = check_device(o)) != ACP_OK) return st;
    hipStream_t sm = static_cast<hipStream_t>(stream);
    uint8_t* d = static_cast<uint8_t*>(device_ptr);
    o->slots[slot].dev = nullptr;
    hipError_t e = hipMemcpyAsync(d + s.off_grads, s.grads.data(), s.grads.size() * sizeof(acp::AwGrad), hipMemcpyHostToDevice, sm);
    if (e == hipSuccess)
      e = hipMemcpyAsync(d + s.off_tiles, s.tiles.data(), s.tiles.size() * sizeof(acp::AwTile), hipMemcpyHostToDevice, sm);
    if (e == hipSuccess) e = hipStreamSynchronize(sm);
    if (e != hipSuccess) return fail(o, ACP_E_DEVICE, std::string("upload failed: ") + hipGetErrorString(e));
    s.tiles = {};  // the device has them
    o->slots[slot].plan = std::move(s);
    o->slots[slot].dev = d;
    o->written.swap(written);
    o->read.swap(read);
    o->err.clear();
    return ACP_OK;
  });
}

acp_status acp_adamw_norm(acp_adamw* o, int32_t slot, float scale, float max_norm, float* clip, void* stream) {
  if (!o) return ACP_E_INVALID;
  return guarded(o, [&]() -> acp_status {
    const acp_status st = check_slot(o, slot);
    if (st != ACP_OK) return st;
    if (!clip || !aligned(clip, 4)) return fail(o, ACP_E_INVALID, "clip must be a device buffer of two floats");
    if (meets(o->written, clip, 8) || meets(o->read, clip, 8))
      return fail(o, ACP_E_INVALID, "clip overlaps the parameters, the state or a slot's block or gradients");
    if (!std::isfinite(scale)) return fail(o, ACP_E_INVALID, "scale must be finite");
    if (!(max_norm > 0.f)) return fail(o, ACP_E_INVALID, "max_norm must be positive (infinity does not clip)");
    const acp_adamw::Slot& s = o->slots[slot];
    acp::AwNormArgs a{};
    a.tensors = reinterpret_cast<const acp::AwTensor*>(o->dev + o->plan.off_tensors);
    a.grads = reinterpret_cast<const acp::AwGrad*>(s.dev + s.plan.off_grads);
    a.tiles = reinterpret_cast<const acp::AwTile*>(s.dev + s.plan.off_tiles);
    a.sums = reinterpret_cast<double*>(s.dev + s.plan.off_sums);
    a.gram = reinterpret_cast<double*>(s.dev + s.plan.off_gram);
    a.clip = clip;
    a.scale = scale;
    a.max_norm = max_norm;
    const hipError_t e = acp::adamw_launch_norm(s.plan, a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return fail(o, ACP_E_DEVICE, std::string("kernel launch failed: ") + hipGetErrorString(e));
    return ACP_OK;
  });
}

acp_status acp_adamw_step(acp_adamw* o, int32_t slot, int64_t step, const acp_adamw_hyper* h, const float* clip,
                          void* stream) {
  if (!o) return ACP_E_INVALID;
  return guarded(o, [&]() -> acp_status {
    const acp_status st = check_slot(o, slot);
    if (st != ACP_OK) return st;
    if (!o->has_params) return fail(o, ACP_E_STATE, "no parameters bound");
    if (step < 1) return fail(o, ACP_E_STEP, "steps count from 1");
    if (!h) return fail(o, ACP_E_INVALID, "null hyperparameters");
    if (!(std::isfinite(h->lr) && h->lr >= 0.0)) return fail(o, ACP_E_INVALID, "lr must be finite and not negative");
    if (!(std::isfinite(h->weight_decay) && h->weight_decay >= 0.0))
      return fail(o, ACP_E_INVALID, "weight_decay must be finite and not negative");
    if (!std::isfinite(h->scale)) return fail(o, ACP_E_INVALID, "scale must be finite");
    acp::AwArgs a{};
    const double t = static_cast<double>(step);
    a.b1 = static_cast<float>(h->beta1);
    a.c1 = static_cast<float>(1.0 - h->beta1);
    a.b2 = static_cast<float>(h->beta2);
    a.c2 = static_cast<float>(1.0 - h->beta2);
    a.lr = static_cast<float>(h->lr / (1.0 - std::pow(h->beta1, t)));
    a.rs = static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(h->beta2, t)));
    a.eps = static_cast<float>(h->eps);
    a.decay = static_cast<float>(1.0 - h->lr * h->weight_decay);
    a.scale = h->scale;
    // as the kernels have them: a beta that fp32 takes for 1 would never let its moment fall
    if (!(h->beta1 >= 0.0 && a.b1 < 1.f) || !(h->beta2 >= 0.0 && a.b2 < 1.f))
      return fail(o, ACP_E_INVALID, "betas must be in [0, 1) and stay below 1 in fp32");
    // (above 2^126 the reciprocal of the update's denominator would be subnormal)
    if (!(a.eps >= 0x1p-126f && a.eps <= 0x1p126f)) return fail(o, ACP_E_INVALID, "eps must be from 2^-126 to 2^126");
    if (!std::isfinite(a.lr)) return fail(o, ACP_E_INVALID, "lr with its bias correction must be finite in fp32");
    if (!std::isfinite(a.decay)) return fail(o, ACP_E_INVALID, "lr times weight_decay must be finite in fp32");
    if (!aligned(clip, 4)) return fail(o, ACP_E_INVALID, "misaligned clip");
    if (clip && meets(o->written, clip, 8))
      return fail(o, ACP_E_INVALID, "clip overlaps the parameters, the state or a slot's block");
    const acp_adamw::Slot& s = o->slots[slot];
    a.tensors = reinterpret_cast<const acp::AwTensor*>(o->dev + o->plan.off_tensors);
    a.grads = reinterpret_cast<const acp::AwGrad*>(s.dev + s.plan.off_grads);
    a.tiles = reinterpret_cast<const acp::AwTile*>(s.dev + s.plan.off_tiles);
    a.m = o->dev + o->plan.off_m;
    a.v = o->dev + o->plan.off_v;
    a.ms = reinterpret_cast<float*>(o->dev + o->plan.off_ms);
    a.vs = reinterpret_cast<float*>(o->dev + o->plan.off_vs);
    a.clip = clip;
    a.key = acp::adamw_step_key(o->plan.seed, step);
    const hipError_t e = acp::adamw_launch_step(s.plan, o->plan.bits, a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return fail(o, ACP_E_DEVICE, std::string("kernel launch failed: ") + hipGetErrorString(e));
    return ACP_OK;
  });
}

const char* acp_adamw_last_error(const acp_adamw* o) { return o ? o->err.c_str() : ""; }

void acp_adamw_destroy(acp_adamw* o) { delete o; }

}  // extern "C"
