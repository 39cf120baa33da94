// Runs the host code of the token-sequence layers on a machine without a GPU, over sizes of all kinds, and prints which kernels it launches and
// which there are: this program defines the runtime calls that the library makes, and the dynamic linker finds them here before the HIP
// runtime's.  No kernel runs, no pointer is read.  A line each: `has <kernel>`, `launched <kernel>`, `bad <what>` (a grid beyond what the hardware
// takes, a status that is not what the sizes ask for); at the end `grid <kernel> <workgroups>` of calls with many empty sequences.
#include <cstdint>
#include <cstdio>
#include <map>
#include <random>
#include <set>
#include <string>

#include "sn_seq.h"

namespace {
struct Dim { uint32_t x, y, z; };
std::map<const void *, std::string> &names() { static std::map<const void *, std::string> m; return m; }
std::set<std::string> launched;
Dim grid, block;
size_t lds;
void *stream;
bool show;
}  // namespace

extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *h; return &h; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { names()[host] = name; }
int __hipPushCallConfiguration(Dim g, Dim b, size_t shared, void *s) { grid = g; block = b; lds = shared; stream = s; return 0; }
int __hipPopCallConfiguration(Dim *g, Dim *b, size_t *shared, void **s) { *g = grid; *b = block; *shared = lds; *s = stream; return 0; }
int hipFuncSetAttribute(const void *, int, int) { return 0; }
int hipGetLastError() { return 0; }
int hipLaunchKernel(const void *f, Dim g, Dim b, void **, size_t, void *)
{
    const std::string &name = names()[f];
    launched.insert(name);
    if (show) std::printf("grid %s %llu\n", name.c_str(), (unsigned long long)g.x * g.y * g.z);
    const uint64_t threads = (uint64_t)g.x * b.x;
    if (!g.x || !g.y || !g.z || threads >= uint64_t(1) << 32 || g.y > 65535 || g.z > 65535) std::printf("bad grid %u %u %u of %s\n", g.x, g.y, g.z, name.c_str());
    return 0;
}
}

namespace {
std::mt19937 rng(11);
int64_t upto(int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); }
template <typename T, size_t N> T one_of(const T (&v)[N]) { return v[rng() % N]; }
void *at(int i) { return reinterpret_cast<void *>(uintptr_t(i + 1) << 44); }
float *fat(int i) { return static_cast<float *>(at(i)); }
void want(sn_status got, const char *what) { if (got != SN_OK) std::printf("bad status %d of %s\n", (int)got, what); }

void conv()
{
    sn_conv1d_shape s = {};
    s.seqs = (int)upto(1, 9);
    s.rows = s.seqs * upto(0, 300);
    s.channels = rng() % 3 ? (int)upto(1, 24) : (int)upto(1, 9000);
    s.width = (int)upto(1, 8);
    s.silu = rng() % 2;
    s.dtype = one_of({SN_F32, SN_BF16});
    s.ld_x = s.ld_y = s.ld_dx = s.channels;
    want(sn_causal_conv1d_fwd(at(0), at(1), fat(2), at(3), &s, nullptr, at(4), at(5), nullptr), "conv fwd");
    const size_t n = sn_causal_conv1d_scratch_bytes(s.rows, s.channels, s.width);
    want(sn_causal_conv1d_bwd(at(0), at(1), fat(2), at(3), at(6), fat(7), fat(8), &s, nullptr, at(4), at(5), at(9), at(10), n, nullptr), "conv bwd");
    want(sn_causal_conv1d_step(at(0), at(1), fat(2), at(3), at(4), at(4), nullptr, 1 << 20, &s, nullptr), "conv step");
}

void heads()
{
    sn_headnorm_shape s = {};
    s.rows = upto(0, 40);
    s.q_heads = rng() % 2 ? (int)upto(1, 4) : (int)upto(1, 80);
    s.k_heads = (int)upto(0, 8);
    s.head_dim = rng() % 2 ? 2 * (int)upto(1, 256) : 16 * (int)upto(1, 32);
    s.rot_dim = rng() % 2 ? 2 * (int)upto(0, s.head_dim / 2) : s.head_dim / 16 * 16 / one_of({1, 2, 4});
    s.rot_dim -= s.rot_dim % 2;
    s.interleaved = rng() % 2;
    s.dtype = one_of({SN_F32, SN_BF16});
    s.eps = 1e-6f;
    s.ld_q = s.ld_yq = s.ld_dq = (int64_t)s.q_heads * s.head_dim;
    s.ld_k = s.ld_yk = s.ld_dk = (int64_t)s.k_heads * s.head_dim;
    const float *freq = s.rot_dim ? fat(4) : nullptr;
    want(sn_headnorm_rot_fwd(at(0), at(1), fat(2), fat(3), nullptr, freq, at(5), at(6), &s, nullptr), "headnorm fwd");
    const size_t n = sn_headnorm_rot_scratch_bytes(s.rows, s.q_heads, s.k_heads, s.head_dim);
    want(sn_headnorm_rot_bwd(at(0), at(1), fat(2), fat(3), nullptr, freq, at(5), at(6), at(7), at(8), fat(9), fat(10), &s, at(11), n, nullptr), "headnorm bwd");
}

void scan()
{
    sn_scan_shape s = {};
    s.seqs = rng() % 4 ? (int)upto(1, 9) : (int)upto(1, 20000);
    s.rows = s.seqs * upto(0, s.seqs < 10 ? 2000 : 40);
    s.groups = (int)upto(1, 4);
    s.channels = s.groups * (rng() % 2 ? (int)upto(1, 40) : 8 * (int)upto(1, 200));
    s.states = rng() % 2 ? (int)upto(1, 64) : one_of({4, 8, 16, 32, 64});
    s.dtype = one_of({SN_F32, SN_BF16});
    s.softplus = rng() % 2;
    s.ragged = rng() % 2;
    s.ld_u = s.ld_dt = s.ld_z = s.ld_y = s.ld_du = s.ld_ddt = s.ld_dz = s.channels;
    s.ld_b = s.ld_c = s.ld_db = s.ld_dc = s.groups * s.states;
    const int32_t *off = s.ragged ? static_cast<const int32_t *>(at(20)) : nullptr;
    size_t least, most;
    float *states = rng() % 2 ? fat(12) : nullptr;
    want(sn_scan_workspace_query(&s, SN_SCAN_FWD, &least, &most), "scan query");
    want(sn_scan_fwd(at(0), at(1), fat(2), at(3), at(4), fat(5), at(6), fat(7), at(8), &s, off, fat(9), fat(10), states, at(11), rng() % 2 ? most : least + (most - least) / 3,
                     nullptr), "scan fwd");
    want(sn_scan_workspace_query(&s, SN_SCAN_BWD, &least, &most), "scan query");
    const size_t own = states ? 0 : sn_scan_states_bytes(&s);
    want(sn_scan_bwd(at(0), at(1), fat(2), at(3), at(4), fat(5), at(6), fat(7), at(8), at(13), at(14), fat(15), at(16), at(17), fat(18), at(19), fat(21), &s, off, fat(9), states,
                     fat(22), fat(23), at(11), own + (rng() % 2 ? most : least), nullptr), "scan bwd");
    want(sn_scan_step(at(0), at(1), fat(2), at(3), at(4), fat(5), at(6), fat(7), at(8), fat(9), fat(9), nullptr, 1 << 20, &s, nullptr), "scan step");
}
}  // namespace

int main()
{
    for (const auto &n : names()) std::printf("has %s\n", n.second.c_str());
    for (int i = 0; i < 20000; ++i) {
        conv();
        heads();
        scan();
    }
    // the largest sizes
    sn_conv1d_shape c = {1 << 30, (1 << 24) - 1, 1, 4, 1, SN_BF16, 1, 1, 1};
    static const int32_t off = 0;
    want(sn_causal_conv1d_fwd(at(0), at(1), nullptr, at(3), &c, &off, at(4), at(5), nullptr), "conv fwd of most rows");
    want(sn_causal_conv1d_bwd(at(0), at(1), nullptr, at(3), at(6), fat(7), fat(8), &c, &off, nullptr, nullptr, at(9), at(10), sn_causal_conv1d_scratch_bytes(c.rows, 1, 4), nullptr),
         "conv bwd of most rows");
    c = {64, 1, 65535 * 256, 4, 1, SN_BF16, 65535 * 256, 65535 * 256, 65535 * 256};
    want(sn_causal_conv1d_bwd(at(0), at(1), nullptr, at(3), at(6), fat(7), fat(8), &c, nullptr, nullptr, nullptr, at(9), at(10),
                              sn_causal_conv1d_scratch_bytes(c.rows, c.channels, 4), nullptr), "conv bwd of most channels");
    sn_headnorm_shape h = {1 << 30, 1, 1, 2, 0, 0, SN_BF16, 1e-6f, 2, 2, 2, 2, 2, 2};
    want(sn_headnorm_rot_bwd(at(0), at(1), nullptr, nullptr, nullptr, nullptr, at(5), at(6), at(7), at(8), fat(9), fat(10), &h, at(11),
                             sn_headnorm_rot_scratch_bytes(h.rows, 1, 1, 2), nullptr), "headnorm bwd of most rows");
    h = {64, 1 << 19, 1 << 19, 2, 0, 0, SN_BF16, 1e-6f, 1 << 20, 1 << 20, 1 << 20, 1 << 20, 1 << 20, 1 << 20};
    want(sn_headnorm_rot_bwd(at(0), at(1), nullptr, nullptr, nullptr, nullptr, at(5), at(6), at(7), at(8), fat(9), fat(10), &h, at(11),
                             sn_headnorm_rot_scratch_bytes(h.rows, h.q_heads, h.k_heads, 2), nullptr), "headnorm bwd of most heads");
    sn_scan_shape z = {1 << 30, (1 << 24) - 1, 1, 1, 1, SN_BF16, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1, 1};
    size_t least, most;
    want(sn_scan_workspace_query(&z, SN_SCAN_BWD, &least, &most), "scan query");
    for (const size_t n : {least, most})
        want(sn_scan_bwd(at(0), at(1), fat(2), at(3), at(4), nullptr, nullptr, nullptr, at(8), at(13), at(14), fat(15), at(16), at(17), nullptr, nullptr, nullptr, &z, &off, fat(9),
                         fat(12), fat(22), fat(23), at(11), n, nullptr), "scan bwd of most rows");
    for (const auto &n : launched) std::printf("launched %s\n", n.c_str());
    // a batch padded with empty sequences
    show = true;
    c = {800, 4096, 2048, 4, 1, SN_BF16, 2048, 2048, 2048};
    want(sn_causal_conv1d_fwd(at(0), at(1), nullptr, at(3), &c, &off, at(4), at(5), nullptr), "conv fwd of empty sequences");
    z = {800, 4096, 2048, 16, 1, SN_BF16, 1, 1, 2048, 2048, 16, 16, 2048, 2048, 2048, 2048, 16, 16, 2048};
    want(sn_scan_workspace_query(&z, SN_SCAN_BWD, &least, &most), "scan query");
    want(sn_scan_fwd(at(0), at(1), fat(2), at(3), at(4), nullptr, nullptr, nullptr, at(8), &z, &off, fat(9), fat(10), nullptr, nullptr, 0, nullptr), "scan fwd of empty sequences");
    want(sn_scan_bwd(at(0), at(1), fat(2), at(3), at(4), nullptr, nullptr, nullptr, at(8), at(13), at(14), fat(15), at(16), at(17), nullptr, nullptr, nullptr, &z, &off, fat(9), fat(12),
                     fat(22), fat(23), at(11), least, nullptr), "scan bwd of empty sequences");
    return 0;
}
