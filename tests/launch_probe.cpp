// Stands in for the runtime's launch calls, so that a process without a GPU can see what the library would launch: loaded with global
// symbols ahead of libconef.so by tests/test_layers_launch.py.  Nothing is launched.
#include <cstdint>
#include <map>
#include <string>
#include <vector>

struct Dim { uint32_t x, y, z; };

namespace {
std::map<const void *, std::string> names;
struct Launch { std::string name; Dim grid, block; };
std::vector<Launch> launches;
Dim pushed_grid, pushed_block;
size_t pushed_shared;
void *pushed_stream;
int dummy;
}  // namespace

extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *p = &dummy; return &p; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { names[host] = name; }
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
int __hipPushCallConfiguration(Dim grid, Dim block, size_t shared, void *stream)
{
    pushed_grid = grid, pushed_block = block, pushed_shared = shared, pushed_stream = stream;
    return 0;
}
int __hipPopCallConfiguration(Dim *grid, Dim *block, size_t *shared, void **stream)
{
    *grid = pushed_grid, *block = pushed_block, *shared = pushed_shared, *stream = pushed_stream;
    return 0;
}
int hipLaunchKernel(const void *f, Dim grid, Dim block, void **, size_t, void *)
{
    launches.push_back({names[f], grid, block});
    return 0;
}
int hipGetLastError() { return 0; }

int probe_kernels() { return (int)names.size(); }
int probe_launches() { return (int)launches.size(); }
const char *probe_launch(int i, uint32_t *out)
{
    const Launch &l = launches[i];
    const uint32_t v[6] = {l.grid.x, l.grid.y, l.grid.z, l.block.x, l.block.y, l.block.z};
    for (int k = 0; k < 6; ++k) out[k] = v[k];
    return l.name.c_str();
}
// kernels' names, one a line
const char *probe_names()
{
    static std::string all;
    all.clear();
    for (const auto &n : names) all += n.second + "\n";
    return all.c_str();
}
void probe_clear() { launches.clear(); }
}
