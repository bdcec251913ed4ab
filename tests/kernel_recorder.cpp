// launch_recorder.cpp that also writes down which kernel a launch is of: the symbol that the library has for it.
#define hipLaunchKernel recorded_launch
#include "launch_recorder.cpp"
#undef hipLaunchKernel

#include <dlfcn.h>
#include <string>

static std::vector<std::string> names;

extern "C" {

int hipLaunchKernel(const void* kernel, Dim3 grid, Dim3 block, void** args, size_t lds, void* stream) {
    Dl_info info;
    names.push_back(dladdr(kernel, &info) && info.dli_sname && info.dli_saddr == kernel ? info.dli_sname : "?");
    return recorded_launch(kernel, grid, block, args, lds, stream);
}
void recorder_names_begin() { names.clear(); }
const char* recorder_name(int i) { return names[i].c_str(); }

}  // extern "C"
