// Stands in front of the runtime (loaded ahead of everything that calls it): notes the names of the kernels that a library registers, and of those
// it launches, which are not run.
#include <dlfcn.h>
#include <stddef.h>

#include <map>
#include <string>

struct Dim {
    unsigned x, y, z;
};

static std::map<const void *, std::string> &names()
{
    static std::map<const void *, std::string> m;
    return m;
}
static std::string launched;

extern "C" {
void __hipRegisterFunction(void **modules, const void *host, char *device, const char *name, unsigned threads, void *tid, void *bid, Dim *block, Dim *grid, int *warp)
{
    using Register = void (*)(void **, const void *, char *, const char *, unsigned, void *, void *, Dim *, Dim *, int *);
    static const Register real = reinterpret_cast<Register>(dlsym(dlopen("libamdhip64.so.7", RTLD_LAZY | RTLD_NOLOAD), "__hipRegisterFunction"));
    names()[host] = name;
    real(modules, host, device, name, threads, tid, bid, block, grid, warp);
}

int hipLaunchKernel(const void *kernel, Dim, Dim, void **, size_t, void *)
{
    launched += names()[kernel] + "\n";
    return 0;
}

const char *registered_kernels(void)
{
    static std::string all;
    all.clear();
    for (const auto &n : names()) all += n.second + "\n";
    return all.c_str();
}

const char *launched_kernels(void) // since the last call
{
    static std::string last;
    last.swap(launched);
    launched.clear();
    return last.c_str();
}
}
