// For the Python binding: addresses of the tensors of a call, where each is what the call takes it for.  In C because a call for a
// single token takes some ten microseconds, and asking a tensor for its type, device, shape and strides from Python a third of one.
//
// A tensor is read through its type's table of C functions, as the DLPack specification (version 1) has them: the function given here
// fills a description of the tensor without owning it.  It needs Python's lock, and so do these calls.
#include <cuda_runtime.h>

#include <cstdint>

namespace {

// DLTensor of the specification.
struct Tensor {
  void* data;
  int32_t device_type, device;
  int32_t dims;
  uint8_t code, bits;
  uint16_t lanes;
  int64_t* shape;
  int64_t* strides;      // in elements
  uint64_t byte_offset;
};
typedef int (*Describe)(void* object, Tensor* out);

constexpr int32_t HOST = 1, CUDA = 2;      // device types

// What the binding has for each argument.
struct Want {
  int32_t code, bits;    // type
  int64_t elements;      // dense: at least so many
  int32_t dense, dims;   // contiguous, whatever the shape; else of this shape and these strides
  int64_t shape[3], strides[3];
};

bool lies_so(const Want& w, const Tensor& t) {
  if (t.dims && !t.strides) return false;
  if (w.dense) {
    int64_t n = 1;
    bool contiguous = true;
    for (int i = t.dims - 1; i >= 0; --i) {
      contiguous = contiguous && (t.shape[i] == 1 || t.strides[i] == n);
      n *= t.shape[i];
    }
    return n >= w.elements && (contiguous || n == 0);
  }
  const int from = t.dims == w.dims - 1 && w.shape[0] == 1;      // (one step: its rows)
  if (t.dims != w.dims - from) return false;
  for (int i = 0; i < t.dims; ++i)
    if (t.shape[i] != w.shape[i + from] || (t.shape[i] > 1 && t.strides[i] != w.strides[i + from])) return false;
  return true;
}

}  // namespace

extern "C" {

// `places`: objects on the way in (`none`: not given), addresses on the way out.  Returns 0, or 1 where an object needs a closer look
// (or has raised); device: -2 the current CUDA device, -1 the host.
int mebptt_binding_places(void* describe, const void* wants, uint64_t* places, int count, int device, uint64_t none) {
  const Want* const w = static_cast<const Want*>(wants);
  if (device != -1 && cudaGetDevice(&device) != cudaSuccess) {
    cudaGetLastError();
    return 1;
  }
  for (int i = 0; i < count; ++i) {
    if (places[i] == none) {
      places[i] = 0;
      continue;
    }
    Tensor t;
    if (reinterpret_cast<Describe>(describe)(reinterpret_cast<void*>(places[i]), &t) != 0) return 1;
    if (t.device_type != (device < 0 ? HOST : CUDA) || (device >= 0 && t.device != device)) return 1;
    if (t.code != w[i].code || t.bits != w[i].bits || t.lanes != 1 || !lies_so(w[i], t)) return 1;
    places[i] = reinterpret_cast<uint64_t>(t.data) + t.byte_offset;
  }
  return 0;
}

}  // extern "C"
