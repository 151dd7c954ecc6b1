// Stand-ins for the HIP runtime under the host side of the operators of include/qoda_matrices.h (csrc/qoda_matrices_api.hip and the launches of
// qoda_mx_quantize.hip, qoda_mx_product.hip and qoda_orthogonal.hip, compiled for the host only): what would be launched is written down, a line a launch, as
//   kernel<arguments> grid.x grid.y grid.z threads first
// and nothing runs.  first: the number of the launch's first workgroup, from the kernel's first argument.
#include <hip/hip_runtime.h>

#include <cxxabi.h>

#include <cstdlib>
#include <map>
#include <string>

#include "../paper_2505_14371_amd/csrc/qoda_matrices.h"

namespace {
std::map<const void *, std::string> &names() {
  static std::map<const void *, std::string> m;
  return m;
}
std::string g_log;
dim3 g_grid, g_block;

std::string plain(const char *mangled) {   // without namespaces, return type and parameters
  int status = 0;
  char *d = abi::__cxa_demangle(mangled, nullptr, nullptr, &status);
  std::string s = d ? d : mangled;
  std::free(d);
  for (const std::string drop : {"void ", "qoda::", "(anonymous namespace)::", " "})
    for (size_t at; (at = s.find(drop)) != std::string::npos;) s.erase(at, drop.size());
  return s.substr(0, s.find('('));
}

template <class Args>
long long first_of(void **args) { return static_cast<const Args *>(args[0])->first; }
}  // namespace

extern "C" {
const char *stand_in_log() { return g_log.c_str(); }
void stand_in_reset() { g_log.clear(); }

void **__hipRegisterFatBinary(const void *) {
  static void *handle;
  return &handle;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *device, unsigned int, uint3 *, uint3 *, dim3 *, dim3 *, int *) { names()[host] = plain(device); }
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) {
  g_grid = grid, g_block = block;
  return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *shared, hipStream_t *stream) {
  *grid = g_grid, *block = g_block, *shared = 0, *stream = nullptr;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void *f, dim3 grid, dim3 block, void **args, size_t, hipStream_t) {
  const std::string name = names()[f];
  const auto is = [&](const char *start) { return name.find(start) == 0; };
  const long long first = is("k_mx_product") || is("k_mx_few_rows") ? first_of<qoda::MxProduct>(args)
                          : is("k_mx_")                             ? first_of<qoda::MxRounding>(args)
                          : is("k_squares") || is("k_start")        ? first_of<qoda::Orthogonal>(args)
                          : is("k_pair_")                           ? first_of<qoda::PairProduct>(args)
                          : is("k_small")                           ? first_of<qoda::SmallOrthogonal>(args)
                                                                    : first_of<qoda::Product>(args);
  g_log += name + " " + std::to_string(grid.x) + " " + std::to_string(grid.y) + " " + std::to_string(grid.z) + " " +
           std::to_string(block.x * block.y * block.z) + " " + std::to_string(first) + "\n";
  return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "stand-in failure"; }

// of the other operators' header, whose host side is not here
extern "C" const char *qoda_operator_error();
}

#include "../paper_2505_14371_amd/csrc/qoda_operators_checks.h"
extern "C" const char *qoda_operator_error() { return qoda::operator_error; }
