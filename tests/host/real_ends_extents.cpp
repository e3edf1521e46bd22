// What the launches of the real-valued ends' calls read and write, without a GPU: this program stands in for the HIP runtime, so that
// every launch of the library's host code arrives here with its arguments.  Checked of each: writes stay within the
// outputs and the workspace that the call asked for, what is read of the workspace was written before and nothing has been written over it
// since, tiles and shares cover every sum once.  Addresses are numbers that nothing dereferences.
// Usage: real_ends_extents cases seed; or real_ends_extents head|grad|matvec followed by sizes of one call (see main()).
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>
#include <vector>

#include "product16.h"
#include "small32.h"

namespace dab {
thread_local int g_last_hip_error = 0;
int ensure_device_ready(int*) { return DAB_OK; }
}  // namespace dab

namespace {
using dab::Product16;
using dab::Small32;
using Address = unsigned long long;

std::map<const void*, std::string>& names() {
    static std::map<const void*, std::string> n;
    return n;
}

struct Range {
    Address at, end;
    const char* name;
    bool inside(const Range& o) const { return at >= o.at && end <= o.end; }
    bool meets(const Range& o) const { return at < o.end && o.at < end; }
};
struct Call {
    std::string text, fault;
    std::vector<Range> inputs, outputs, kept;    // kept: pieces of the workspace that hold what was written
    Range ws{};
    int launches = 0;
} now;

void fault(const std::string& kernel, const char* what, const Range* r = nullptr) {
    if (!now.fault.empty()) return;
    now.fault = std::string(what) + " (launch " + std::to_string(now.launches) + ", " + kernel.substr(0, 60) + ")";
    if (r) now.fault += std::string(": ") + r->name + ", " + std::to_string(static_cast<long long>(r->end - now.ws.end)) + " bytes past the workspace of " + std::to_string(now.ws.end - now.ws.at);
}
Range range(const void* p, unsigned long long bytes, const char* name) { return {reinterpret_cast<Address>(p), reinterpret_cast<Address>(p) + bytes, name}; }

void write(const std::string& k, Range r) {
    for (const Range& o : now.outputs)
        if (r.inside(o)) return;
    if (!r.inside(now.ws)) return fault(k, "writes outside the workspace and the outputs", &r);
    for (size_t i = 0; i < now.kept.size();)
        if (now.kept[i].meets(r)) now.kept.erase(now.kept.begin() + static_cast<long>(i));
        else ++i;
    now.kept.push_back(r);
}
void read(const std::string& k, Range r) {
    for (const Range& o : now.inputs)
        if (r.inside(o)) return;
    for (const Range& o : now.kept)
        if (r.inside(o)) return;
    fault(k, "reads what no input and no earlier launch holds", &r);
}

// The whole numbers of a kernel's template arguments.
std::vector<int> numbers(const std::string& name) {
    std::vector<int> v;
    const size_t from = name.find("kernelI");
    for (size_t i = from == std::string::npos ? name.size() : from; i + 2 < name.size(); ++i)
        if (name[i] == 'L' && (name[i + 1] == 'i' || name[i + 1] == 'b')) v.push_back(std::atoi(name.c_str() + i + 2));
    return v;
}

void operand(const std::string& k, const dab::Operand16& o, bool rows_inner, long long rows, long long K, int size, uint32_t segs, int n_seg, const char* name) {
    for (int s = 0; s < n_seg; ++s) {
        const long long plane = (segs >> (4 * s) & 15) * o.plane, n = rows_inner ? rows : K, far = rows_inner ? K : rows;
        const long long words = size == 4 ? n * 4 : (n + 1) / 2 * 4;
        read(k, range(static_cast<const char*>(o.p) + plane * size, static_cast<unsigned long long>((far - 1) * o.ld * size + words), name));
    }
}

void product(const std::string& k, const std::vector<int>& t, const Product16& g, dim3 grid, dim3 block) {
    const int epi = t[0], TM = t[1], TN = t[2], WM = t[3], WN = t[4];
    const bool ends = k.find("ends_kernel") != std::string::npos, wide = k.find("product32") != std::string::npos;
    const bool arc = t.size() > 5 && t[5], brc = t.size() > 6 && t[6];
    const int size = wide ? 4 : 2, step = 128 / size, M = g.M, N = g.N;
    const long long tiles = 1ll * g.tiles_m * g.tiles_n;
    if (1ll * g.tiles_m * TM < M || 1ll * (g.tiles_m - 1) * TM >= M || 1ll * g.tiles_n * TN < N || 1ll * (g.tiles_n - 1) * TN >= N) fault(k, "tiles do not cover the result");
    if (g.steps != g.n_seg * ((g.K + step - 1) / step) || g.whole + g.rest != tiles) fault(k, "steps or tiles");
    if (8ll * g.whole_xcd < g.whole || 8ll * g.rest_xcd < 1ll * g.rest * g.shares) fault(k, "tiles that no workgroup takes");
    if (grid.x != 8u * static_cast<unsigned>(g.whole_xcd + g.rest_xcd) || block.x != 64u * static_cast<unsigned>(WM * WN)) fault(k, "grid");
    if (g.rest == 0 && g.shares != 1) fault(k, "shares of nothing");
    operand(k, g.A, arc, M, g.K, size, g.seg_a, g.n_seg, "A");
    operand(k, g.B, brc, N, g.K, size, g.seg_b, g.n_seg, "B");
    if (epi == dab::kEpiStore) {
        if (g.shares > 1) write(k, range(g.part, 1ull * g.rest * g.shares * TM * TN * 4, "sums of shares"));
        if (g.rest && (g.share_steps < 1 || 1ll * g.share_steps * g.shares < g.steps || 1ll * g.share_steps * (g.shares - 1) >= g.steps)) fault(k, "shares that do not cover the sum once");
        if (g.add) read(k, range(g.add, 4ull * M * N, "sums of the pieces before"));
        if (g.targets) read(k, range(g.targets, 8ull * M, "targets"));
        if (g.factor) read(k, range(g.factor, 8, "weights' factor"));
        if (g.whole || g.shares == 1) write(k, range(g.C, (1ull * (M - 1) * static_cast<unsigned long long>(g.ldc) + N) * (g.out_bf16 ? 2 : 4), "result"));
        return;
    }
    // (a softmax needs its sum whole: one workgroup a tile, or a quarter of a tile where the kernel has them)
    if (g.rest && !(ends && TM == 256 && g.shares == 4)) fault(k, "a softmax in shares");
    read(k, range(g.targets, 8ull * M, "targets"));
    if (epi == dab::kEpiStats) {
        write(k, range(g.stats, 8ull * g.tiles_n * WN * M, "statistics"));
        write(k, range(g.target_logit, 4ull * M, "targets' logits"));
    } else {
        read(k, range(g.lse, 4ull * M, "lse"));
        if (g.g) read(k, range(g.g, 4ull * M, "weights"));
        if (g.factor) read(k, range(g.factor, 8, "weights' factor"));
        if (1ll * g.tiles_n * TN > g.ldp) fault(k, "rows of P that run into each other");
        const unsigned long long elems = 1ull * (g.p_planes - 1) * static_cast<unsigned long long>(g.p_plane) + 1ull * (M - 1) * static_cast<unsigned long long>(g.ldp) + 1ull * g.tiles_n * TN;
        write(k, range(g.P, elems * size, "P"));
    }
}
void small(const std::string& k, const Small32& g, int size_a, bool arc, int size_b, bool brc) {
    auto side = [&](const dab::Source32& o, int rows, int size, bool rc, const char* name) {
        const unsigned long long far = rc ? g.K : rows, n = rc ? rows : g.K;
        read(k, range(o.p, ((far - 1) * static_cast<unsigned long long>(o.ld) + n) * size, name));
    };
    side(g.A, g.M, size_a, arc, "A");
    side(g.B, g.N, size_b, brc, "B");
}

template <typename T>
T argument(void** args, int i) { return *static_cast<T*>(args[i]); }

void launched(const void* f, dim3 grid, dim3 block, void** a) {
    const std::string k = names().count(f) ? names()[f] : "unknown";
    ++now.launches;
    auto is = [&](const char* n) { return k.find(n) != std::string::npos; };
    const std::vector<int> t = numbers(k);
    const bool f32 = is("kernelIf");
    if (is("product16_") || is("product32_")) {
        product(k, t, argument<Product16>(a, 0), grid, block);
    } else if (is("join16_kernel")) {
        const Product16 g = argument<Product16>(a, 0);
        read(k, range(g.part, 1ull * g.rest * g.shares * t[0] * t[1] * 4, "sums of shares"));
        if (g.add) read(k, range(g.add, 4ull * g.M * g.N, "sums of the pieces before"));
        write(k, range(g.C, (1ull * (g.M - 1) * static_cast<unsigned long long>(g.ldc) + g.N) * (g.out_bf16 ? 2 : 4), "result"));
    } else if (is("planes16_kernel")) {
        const unsigned long long rows = argument<int>(a, 1), cols = argument<int>(a, 2), ld = argument<int64_t>(a, 3), ldp = argument<int>(a, 8), size = f32 ? 4 : 2;
        read(k, range(argument<void*>(a, 0), ((rows - 1) * ld + cols) * size, "rows"));
        write(k, range(argument<void*>(a, 7), t.back() * rows * ldp * 2, "planes"));
        if (void* factor = argument<void*>(a, 12)) {
            if (grid.x != argument<unsigned>(a, 10) + 1) fault(k, "no workgroup for the factor");
            read(k, range(argument<void*>(a, 11), 4 * rows, "weights"));
            write(k, range(factor, 8, "weights' factor"));
        } else if (grid.x != argument<unsigned>(a, 10)) {
            fault(k, "grid");
        }
    } else if (is("rows32_kernel")) {
        const unsigned long long ldp = argument<int>(a, 7);
        write(k, range(argument<void*>(a, 6), 16ull * argument<int64_t>(a, 8), "rows"));
        if (argument<int64_t>(a, 8) % static_cast<int64_t>(ldp / 4)) fault(k, "rows");
    } else if (is("head_join_kernel")) {
        const unsigned long long T = argument<int>(a, 4), blocks = argument<int>(a, 6);
        read(k, range(argument<void*>(a, 0), blocks * T * 8, "statistics"));
        read(k, range(argument<void*>(a, 1), T * 4, "targets' logits"));
        write(k, range(argument<void*>(a, 7), T * 4, "loss"));
        write(k, range(argument<void*>(a, 8), T * 4, "lse"));
    } else if (is("head_unstack_kernel")) {
        const unsigned long long n = argument<int>(a, 1);
        read(k, range(argument<void*>(a, 0), 8 * n, "sums of both planes"));
        read(k, range(argument<void*>(a, 4), 8 * (n / argument<int>(a, 3)), "targets"));
        write(k, range(argument<void*>(a, 2), 2 * n, "dH"));
    } else if (is("small_stats_kernel") || is("small_softmax_kernel")) {
        const Small32 g = argument<Small32>(a, 0);
        small(k, g, f32 ? 4 : 2, false, f32 ? 4 : 2, false);
        if (is("stats")) {
            write(k, range(g.stats, 8ull * ((g.N + 31) / 32) * g.M, "statistics"));
            write(k, range(g.target_logit, 4ull * g.M, "targets' logits"));
        } else {
            write(k, range(g.C, 4ull * (static_cast<unsigned long long>(g.M - 1) * g.ldc + g.N), "P"));
        }
    } else if (is("small_gradients_kernel")) {
        for (int i = 0; i < 2; ++i) {
            const Small32 g = argument<Small32>(a, i);
            small(k, g, 4, i == 0, f32 ? 4 : 2, true);
            if (g.targets) read(k, range(g.targets, 8ull * g.M, "targets"));
            write(k, range(g.C, (g.dtype == DAB_F32 ? 4ull : 2ull) * (static_cast<unsigned long long>(g.M - 1) * g.ldc + g.N), "result"));
        }
    } else if (is("grad_operands_kernel")) {
        const unsigned long long rows = argument<int>(a, 6), ldp = argument<int>(a, 10);
        write(k, range(argument<void*>(a, 3), 16ull * argument<int64_t>(a, 2), "saved input"));
        if (argument<unsigned>(a, 4) < grid.x) write(k, range(argument<void*>(a, 9), t.back() * rows * ldp * 2, "planes"));
    } else if (is("w4_tokens_kernel")) {
        const unsigned long long Kt = argument<int>(a, 4), tiles = argument<int>(a, 7);
        write(k, range(argument<void*>(a, 8), grid.y * Kt * 4 * tiles * 1024, "tokens"));
    } else if (!is("w4_matvec_kernel")) {
        fault(k, "a kernel that this program does not know");
    }
}
}  // namespace

// ---------------------------------------------------------------- the runtime that the library's host code finds
extern "C" {
void** __hipRegisterFatBinary(const void*) {
    static void* module = nullptr;
    return &module;
}
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* f, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { names()[f] = name; }
void __hipRegisterVar(void**, void*, char*, const char*, int, size_t, int, int) {}
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
    launched(f, grid, block, args);
    return hipSuccess;
}
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
}

namespace {
uint64_t g_state = 1;
double uniform() {
    g_state = g_state * 6364136223846793005ull + 1442695040888963407ull;
    return static_cast<double>(g_state >> 11) / 9007199254740992.0;
}
int whole(int lo, int hi) {      // spread over the logarithm; often a round number, often not
    int v = static_cast<int>(std::lround(std::exp(std::log(lo) + uniform() * (std::log(hi) - std::log(lo)))));
    if (uniform() < 0.5 && v >= 32) v = 16 * ((v + 8) / 16);
    return v < lo ? lo : v > hi ? hi : v;
}

// Regions of addresses far apart.
Range region(int i, unsigned long long bytes, const char* name) { return {(1ull + i) << 44, ((1ull + i) << 44) + bytes, name}; }
void* at(const Range& r) { return reinterpret_cast<void*>(r.at); }

int finish(int rc) {
    if (rc != DAB_OK && now.fault.empty()) now.fault = "status " + std::to_string(rc);
    if (now.launches == 0 && now.fault.empty()) now.fault = "no launch";
    if (now.fault.empty()) return 0;
    std::printf("%s: %s\n", now.text.c_str(), now.fault.c_str());
    return 1;
}
void begin(const std::string& text, std::vector<Range> inputs, std::vector<Range> outputs, unsigned long long ws) {
    now = Call{};
    now.text = text, now.inputs = std::move(inputs), now.outputs = std::move(outputs), now.ws = region(12, ws, "workspace");
}

int head(int T, int D, int V, int dtype, long long ldh, long long ldw, bool all = true) {
    const unsigned long long size = dtype == DAB_F32 ? 4 : 2;
    const Range H = region(0, ((T - 1) * static_cast<unsigned long long>(ldh) + D) * size, "H"), W = region(1, ((V - 1) * static_cast<unsigned long long>(ldw) + D) * size, "W");
    const Range targets = region(2, 8ull * T, "targets"), lse = region(3, 4ull * T, "lse"), g = region(4, 4ull * T, "g"), loss = region(5, 4ull * T, "loss");
    const Range dH = region(6, 1ull * T * D * size, "dH"), dW = region(7, 1ull * V * D * size, "dW");
    char text[160];
    std::snprintf(text, sizeof text, "head %d x %d -> %d, type %d, rows %lld and %lld apart", T, D, V, dtype, ldh, ldw);
    int bad = 0;
    if (all) {
        const size_t n = dab_head_loss_workspace_bytes(T, D, V, dtype, ldh, ldw);
        begin(std::string(text) + ", loss", {H, W, targets}, {loss, lse}, n);
        bad += finish(dab_head_loss(at(H), ldh, at(W), ldw, dtype, static_cast<int64_t*>(at(targets)), -100, T, D, V, static_cast<float*>(at(loss)),
                                    static_cast<float*>(at(lse)), at(now.ws), n, nullptr));
    }
    const size_t n = dab_head_loss_gradient_workspace_bytes(T, D, V, dtype, ldh, ldw);
    begin(std::string(text) + ", gradient", {H, W, targets, lse, g}, {dH, dW}, n);
    bad += finish(dab_head_loss_gradient(at(H), ldh, at(W), ldw, dtype, static_cast<int64_t*>(at(targets)), -100, static_cast<float*>(at(lse)),
                                         static_cast<float*>(at(g)), T, D, V, at(dH), at(dW), at(now.ws), n, nullptr));
    return bad;
}
int grad(int rows, int cols, int F, int dtype, long long lddy) {
    const unsigned long long size = dtype == DAB_F32 ? 4 : 2, groups = (cols + 31ull) / 32;
    const Range dY = region(0, ((rows - 1) * static_cast<unsigned long long>(lddy) + F) * size, "dY"), Q = region(1, rows * groups * 32, "Q"), S = region(2, rows * groups, "S");
    const Range dW = region(3, 4ull * F * cols, "dW");
    char text[160];
    std::snprintf(text, sizeof text, "weight gradient, %d rows %d -> %d, type %d, rows %lld apart", rows, cols, F, dtype, lddy);
    const size_t n = dab_ckpt8_weight_gradient_workspace_bytes(rows, cols, F, dtype, lddy);
    begin(text, {dY, Q, S}, {dW}, n);
    return finish(dab_ckpt8_weight_gradient(at(dY), dtype, lddy, static_cast<int8_t*>(at(Q)), static_cast<uint8_t*>(at(S)), rows, cols, F,
                                            static_cast<float*>(at(dW)), at(now.ws), n, nullptr));
}
int matvec(int B, int K, int F, int dtype, long long ldx) {
    const unsigned long long size = dtype == DAB_F32 ? 4 : 2;
    const Range X = region(0, ((B - 1) * static_cast<unsigned long long>(ldx) + K) * size, "X"), Y = region(1, 1ull * B * F * size, "Y");
    char text[160];
    std::snprintf(text, sizeof text, "4-bit product, %d tokens %d -> %d, type %d, rows %lld apart", B, K, F, dtype, ldx);
    const size_t n = dab_w4_matvec_workspace_bytes(B, K, F, dtype, ldx);
    begin(text, {X}, {Y}, n);
    return finish(dab_w4_matvec(at(X), dtype, ldx, reinterpret_cast<uint8_t*>(1ull << 47), reinterpret_cast<uint8_t*>(3ull << 47), B, K, F, at(Y), n ? at(now.ws) : nullptr, n, nullptr));
}
// Launches of 2^32 threads along a dimension are refused, those of fewer are not.
void kernel_of_nothing() {}
int too_many_threads() {
    int bad = 0;
    for (const dim3 grid : {dim3(1u << 24), dim3(1, 1u << 24), dim3((1u << 24) + 3, 2), dim3(0xffffffffu)}) {
        now = Call{};
        bad += dab::launch(kernel_of_nothing, grid, dim3(256, 256), 0, nullptr) != DAB_ERR_UNSUPPORTED || now.launches != 0;
    }
    now = Call{};
    bad += dab::launch(kernel_of_nothing, dim3((1u << 24) - 1, 65535), dim3(256), 0, nullptr) != DAB_OK || now.launches != 1;
    if (bad) std::printf("launches of too many threads: %d\n", bad);
    return bad;
}
// A plan whose shares have less room than they need is refused before anything is launched.
int refusal() {
    const dab::Plan16 pl = dab::plan16(300, 300, 100000, 1, dab::kAnyShares16);
    Product16 g{};
    g.M = g.N = 300, g.K = 100000, g.n_seg = 1;
    now = Call{};
    const int rc = dab::launch16(dab::kEpiStore, true, true, g, pl, pl.part_bytes - 1, nullptr);
    if (pl.shares > 1 && pl.part_bytes > 0 && rc == DAB_ERR_UNSUPPORTED && now.launches == 0) return 0;
    std::printf("shares without room: status %d, %d launches\n", rc, now.launches);
    return 1;
}
}  // namespace

int main(int argc, char** argv) {
    auto num = [&](int i) { return i < argc ? std::atoi(argv[i]) : 0; };
    if (argc > 1 && !std::strcmp(argv[1], "head")) {         // T D V type, any number of times
        int bad = 0;
        for (int i = 2; i + 3 < argc; i += 4) bad += head(num(i), num(i + 1), num(i + 2), num(i + 3), num(i + 1), num(i + 1));
        return bad != 0;
    }
    const int cases = argc > 1 ? num(1) : 20000;
    g_state = 977ull * static_cast<unsigned long long>(argc > 2 ? num(2) : 1) + 1;
    int bad = refusal() + too_many_threads();
    for (int i = 0; i < cases; ++i) {
        const int T = whole(1, 32768), D = whole(1, 16384), V = whole(1, 262144), dtype = uniform() < 0.6 ? DAB_BF16 : DAB_F32;
        auto apart = [&](int n) { return uniform() < 0.7 ? static_cast<long long>(n) : n + whole(1, 200); };
        bad += head(T, D, V, dtype, apart(D), apart(D));
        const int rows = whole(1, 1 << 20), cols = whole(1, 16384), F = whole(1, 16384);
        bad += grad(rows, cols, F, static_cast<int>(uniform() * 3), apart(F));
        const int B = whole(1, 4096), K = whole(1, 65536), N = whole(1, 262144);
        bad += matvec(B, K, N, static_cast<int>(uniform() * 3), apart(K));
    }
    // usual widths, vocabularies and batches
    static const int kT[] = {64, 128, 256, 512, 1024, 2048, 4096, 6144, 8192, 16384, 32768};
    static const int kD[] = {512, 1024, 2048, 2560, 4096, 5120, 6144, 7168, 8192, 16384};
    static const int kV[] = {32000, 32768, 50257, 50304, 65536, 100352, 128000, 128256, 131072, 151936, 256000};
    for (const int T : kT)
        for (const int D : kD)
            for (const int V : kV)
                for (const int dtype : {DAB_BF16, DAB_F32}) bad += head(T, D, V, dtype, D, D);
    std::printf("%d cases, %d faults\n", cases, bad);
    return bad != 0;
}
