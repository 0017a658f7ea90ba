// Stands in for the HIP runtime in a process without a GPU: loaded before the
// library, it takes the library's launches and writes down what each was given,
// one line of JSON per launch.  Nothing runs; every call succeeds.
#include <cxxabi.h>
#include <stdint.h>
#include <stdlib.h>

#include <map>
#include <string>

#include "linear_common.h"

#define SHOWN extern "C" __attribute__((visibility("default")))

namespace {

std::map<const void*, std::string>& names() {
  static std::map<const void*, std::string> m;
  return m;
}
std::string text;

struct Config {
  dim3 grid, block;
  size_t shared;
  hipStream_t stream;
} config;

// As in linear.hip.
struct Copy {
  const void* from;
  void* to;
  int64_t ld, to_ld, lines;
  int len;
};

// As in gradclip.hip.
struct List {
  const void* g[240];
  void* out[240];
  int64_t n[240];
  int first[241];
  unsigned char dtype[240];
  int count, chunk;
};

void put(const char* key, int64_t v) { text += ", \"" + std::string(key) + "\": " + std::to_string(v); }
void put(const char* key, const void* p) { put(key, (int64_t)(uintptr_t)p); }

void put(const linear::Product& p) {
  put("A", p.A), put("B", p.B), put("lda", p.lda), put("ldb", p.ldb), put("M", p.M), put("N", p.N), put("K", p.K);
  put("arows", p.arows), put("aK", p.aK), put("brows", p.brows), put("bK", p.bK), put("splits", p.splits), put("part", p.part);
  put("C", p.e.C), put("ldc", p.e.ldc);
}

void put(const char* which, const Copy& c) {
  const std::string w = which;
  put((w + "from").c_str(), c.from), put((w + "to").c_str(), c.to), put((w + "ld").c_str(), c.ld);
  put((w + "to_ld").c_str(), c.to_ld), put((w + "lines").c_str(), c.lines), put((w + "len").c_str(), (int64_t)c.len);
}

}  // namespace

SHOWN void** __hipRegisterFatBinary(const void*) {
  static void* one = nullptr;
  return &one;
}
SHOWN void __hipRegisterFunction(void**, const void* host, char*, const char* device, unsigned, void*, void*, dim3*, dim3*, int*) {
  // the demangler does not know the 16-bit types: bf16 is shown as "unsigned
  // short", fp16 as "short"
  std::string name = device;
  for (size_t at; (at = name.find("DF16b")) != std::string::npos;) name.replace(at, 5, "t");
  for (size_t at; (at = name.find("DF16_")) != std::string::npos;) name.replace(at, 5, "s");
  char* plain = abi::__cxa_demangle(name.c_str(), nullptr, nullptr, nullptr);
  if (plain) name = plain;
  free(plain);
  const std::string space = "linear::(anonymous namespace)::";
  for (size_t at; (at = name.find(space)) != std::string::npos;) name.erase(at, space.size());
  names()[host] = name;
}
SHOWN void __hipRegisterVar(void**, void*, char*, const char*, int, size_t, int, int) {}
SHOWN void __hipUnregisterFatBinary(void**) {}

SHOWN hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, hipStream_t stream) {
  config = Config{grid, block, shared, stream};
  return hipSuccess;
}
SHOWN hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, hipStream_t* stream) {
  *grid = config.grid, *block = config.block, *shared = config.shared, *stream = config.stream;
  return hipSuccess;
}

SHOWN hipError_t hipGetDevice(int* dev) {
  *dev = 0;
  return hipSuccess;
}
SHOWN hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t a, int) {
  *v = a == hipDeviceAttributeMultiprocessorCount ? 256 : 0;
  return hipSuccess;
}
SHOWN hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
SHOWN hipError_t hipGetLastError() { return hipSuccess; }

SHOWN hipError_t hipLaunchKernel(const void* host, dim3 grid, dim3 block, void** args, size_t lds, hipStream_t) {
  const std::string name = names()[host];
  text += "{\"kernel\": \"" + name + "\"";
  put("grid", (int64_t)grid.x * grid.y * grid.z), put("block", (int64_t)block.x), put("lds", (int64_t)lds);
  auto is = [&](const char* part) { return name.find(part) != std::string::npos; };
  if (is("ring_kernel") || is("wide_kernel") || is("join_kernel")) put(*static_cast<const linear::Product*>(args[0]));
  if (is("pad_kernel")) {
    put("a_", *static_cast<const Copy*>(args[0]));
    put("b_", *static_cast<const Copy*>(args[1]));
    put("a_blocks", (int64_t)*static_cast<const int*>(args[2]));
  }
  if (is("slope_kernel")) {      // kn, t, span, dO, lddo, Z, ldz, act, dZ, lddz, part, dbias
    put("kn", (int64_t)*static_cast<const int*>(args[0])), put("t", (int64_t)*static_cast<const int*>(args[1]));
    put("span", (int64_t)*static_cast<const int*>(args[2]));
    put("dZ", *static_cast<void* const*>(args[8])), put("lddz", *static_cast<const int64_t*>(args[9]));
    put("part", *static_cast<void* const*>(args[10])), put("dbias", *static_cast<void* const*>(args[11]));
  }
  if (is("norm_kernel") || is("scale_kernel")) {
    const List& l = *static_cast<const List*>(args[0]);
    put("count", (int64_t)l.count), put("chunk", (int64_t)l.chunk);
    // the chunks of each tensor, by the numbers before it and before the next
    text += ", \"chunks\": [";
    for (int i = 0; i < l.count; ++i) text += (i ? ", " : "") + std::to_string((int64_t)l.first[i + 1] - l.first[i]);
    text += "], \"last\": " + std::to_string(l.first[l.count]);
  }
  text += "}\n";
  return hipSuccess;
}

// What was launched since the last call.
SHOWN const char* recorded() {
  static std::string given;
  given.swap(text);
  text.clear();
  return given.c_str();
}
