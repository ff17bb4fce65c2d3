// One operation on the caller's device memory and stream (ooc_run_fn): the signature checks of a
// registered function, then checks of the addresses, then the same launches.  Nothing is kept
// between calls, allocated on the device or waited for, so a call can be recorded into a graph.
#include <string>

#include "kernels.h"

namespace ooc {

namespace {

// Makes `device` current for the scope, the caller's device again behind it.
class DeviceScope {
 public:
  explicit DeviceScope(int device) {
    status = hipGetDevice(&before_);
    if (status == hipSuccess && before_ != device) {
      status = hipSetDevice(device);
      changed_ = status == hipSuccess;
    }
  }
  ~DeviceScope() {
    if (changed_) (void)hipSetDevice(before_);
  }
  hipError_t status;

 private:
  int before_ = 0;
  bool changed_ = false;
};

}  // namespace

ooc_status run_fn(int32_t device, hipStream_t stream, int32_t op, void* const* ptrs,
                  const uint64_t* bytes, const uint8_t* access, int32_t n, const int64_t* attrs,
                  int32_t n_attrs, std::string* err) {
  auto refuse = [&](ooc_status s, const std::string& why) {
    *err = "ooc_run_fn: " + why;
    return s;
  };
  if (n <= 0 || !ptrs || !bytes || !access) return refuse(OOC_E_INVALID, "a function needs variables");
  if (n_attrs < 0 || (n_attrs > 0 && !attrs)) return refuse(OOC_E_INVALID, "bad attributes");
  if (device < 0) return refuse(OOC_E_INVALID, "bad device");
  if (op == OOC_OP_SGD)
    return refuse(OOC_E_UNSUPPORTED, "SGD takes its rates from ooc_step and runs there alone");
  Fn fn;
  fn.op = op;
  fn.attrs.assign(attrs, attrs + n_attrs);
  std::vector<Var> vars((size_t)n);
  for (int32_t j = 0; j < n; ++j) {
    const auto at = reinterpret_cast<uintptr_t>(ptrs[j]);
    const std::string which = "variable " + std::to_string(j);
    if (access[j] < OOC_R || access[j] > OOC_RW) return refuse(OOC_E_INVALID, "bad access flag");
    if (!at || at % 16) return refuse(OOC_E_INVALID, which + " is NULL or not aligned to 16 bytes");
    if (bytes[j] == 0 || bytes[j] > (1ull << 50))
      return refuse(OOC_E_INVALID, which + " has a bad size");
    for (int32_t k = 0; k < j; ++k) {
      const auto other = reinterpret_cast<uintptr_t>(ptrs[k]);
      if (((access[j] | access[k]) & OOC_W) && at < other + bytes[k] && other < at + bytes[j])
        return refuse(OOC_E_INVALID, which + " overlaps variable " + std::to_string(k) +
                                         " and one of them is written");
    }
    vars[j] = Var{bytes[j], OOC_TEMP};
    fn.vars.push_back(FnVar{j, access[j]});
  }
  const std::string e = check_fn(vars, fn);
  if (!e.empty()) return refuse(OOC_E_INVALID, e);

  DeviceScope scope(device);
  if (scope.status != hipSuccess) {
    (void)hipGetLastError();
    return refuse(OOC_E_DEVICE, "HIP device " + std::to_string(device) + " is not available: " +
                                    hipGetErrorString(scope.status));
  }
  int of = device;
  if (stream && (hipStreamGetDevice(stream, &of) != hipSuccess || of != device)) {
    (void)hipGetLastError();
    return refuse(OOC_E_INVALID, "the stream is not one of device " + std::to_string(device));
  }
  for (int32_t j = 0; j < n; ++j) {
    hipPointerAttribute_t a;
    hipDeviceptr_t base = nullptr;
    size_t size = 0;
    if (hipPointerGetAttributes(&a, ptrs[j]) != hipSuccess || a.type != hipMemoryTypeDevice ||
        a.device != device || hipMemGetAddressRange(&base, &size, ptrs[j]) != hipSuccess) {
      (void)hipGetLastError();
      return refuse(OOC_E_INVALID, "variable " + std::to_string(j) +
                                       " is not device memory of device " + std::to_string(device));
    }
    const uint64_t off = (uint64_t)(static_cast<char*>(ptrs[j]) - static_cast<char*>(base));
    if (off > size || bytes[j] > size - off)
      return refuse(OOC_E_INVALID, "variable " + std::to_string(j) + " is longer than its memory");
  }
  const std::vector<uint8_t> dead((size_t)n, 0);   // the caller may read whatever is written
  // The launchers ask hipGetLastError, which would also report an error that an earlier call of the
  // caller's left pending; there is no way to put one back.
  (void)hipGetLastError();
  const hipError_t r = launch_fn(fn, ptrs, bytes, dead.data(), Join::kNone, BnBehind{}, 0.f, 0.f,
                                 stream);
  if (r != hipSuccess) return refuse(OOC_E_DEVICE, std::string("launch failed: ") + hipGetErrorString(r));
  return OOC_OK;
}

}  // namespace ooc
