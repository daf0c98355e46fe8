// The built library on a HIP runtime of host memory: this program defines the
// runtime's functions that the library calls, opens the library, and sees what
// it would launch.  (No device is touched and no kernel runs.)  Modes:
//   alias LIB            "name status" of calls whose buffers overlap or touch
//   attributes LIB       two threads' first calls of the scorer's backward pass:
//                        "EARLY name" of each kernel launched before its
//                        attribute was set, then "launches N"
//   creation LIB LENGTHS...              "mallocs N copies N" of crf_plan_create
//   memory LIB LENGTHS...                crf_plan_create with host memory that runs out
//                        after 0, 1, 2, ... allocations: "status N times N" of each
//                        status in a row, "left N" device allocations never freed
//   launches LIB CALL FLAGS LENGTHS...   the kernels of a call in order, "K name",
//                        and "A sentences pointer" of one that marks log Z as missing
#include <cxxabi.h>
#include <dlfcn.h>
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <atomic>
#include <chrono>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <mutex>
#include <new>
#include <set>
#include <string>
#include <thread>
#include <vector>

#include "crf_inside.h"

namespace {
std::mutex mu;
std::map<const void *, std::string> names;
std::set<const void *> ready;       // functions whose LDS attribute is set
std::vector<std::string> launched, early, marked;
void *const workspace = reinterpret_cast<void *>((uintptr_t)9 << 40);
int mallocs = 0, frees = 0, copies = 0;
thread_local int64_t news_left = -1;   // host allocations until one fails; -1: none does
bool slow_attributes = false, watch_attributes = false;
struct Config {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
};
thread_local Config config;
}  // namespace

// (the library's allocations too)
void *operator new(size_t n) {
    if (news_left == 0) throw std::bad_alloc();
    if (news_left > 0) --news_left;
    void *p = std::malloc(n ? n : 1);
    if (p == nullptr) throw std::bad_alloc();
    return p;
}
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, size_t) noexcept { std::free(p); }

extern "C" {
void **__hipRegisterFatBinary(const void *) {
    static void *handle;
    return &handle;
}
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *host, char *, const char *name, unsigned, void *, void *, dim3 *, dim3 *, int *) {
    int st = 0;
    char *d = abi::__cxa_demangle(name, nullptr, nullptr, &st);
    names[host] = st == 0 ? d : name;
    std::free(d);
}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t lds, hipStream_t s) {
    config = Config{g, b, lds, s};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *g, dim3 *b, size_t *lds, hipStream_t *s) {
    *g = config.grid;
    *b = config.block;
    *lds = config.lds;
    *s = config.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *f, dim3, dim3, void **args, size_t lds, hipStream_t) {
    std::lock_guard<std::mutex> lock(mu);
    launched.push_back(names[f]);
    if (names[f].find("mark_missing") != std::string::npos) {   // (ids, how many, log Z)
        const int32_t *ids = *static_cast<const int32_t **>(args[0]);
        std::string a = "A";
        for (int k = 0; k < *static_cast<int *>(args[1]); ++k) a += " " + std::to_string(ids[k]);
        marked.push_back(a + (*static_cast<void **>(args[2]) == workspace ? " workspace" : " elsewhere"));
    }
    if (watch_attributes && lds > 65536 && ready.count(f) == 0) early.push_back(names[f]);
    return hipSuccess;
}
hipError_t hipFuncSetAttribute(const void *f, hipFuncAttribute, int) {
    if (slow_attributes) std::this_thread::sleep_for(std::chrono::milliseconds(2));
    std::lock_guard<std::mutex> lock(mu);
    ready.insert(f);
    return hipSuccess;
}
hipError_t hipGetDevice(int *d) {
    *d = 0;
    return hipSuccess;
}
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipDeviceGetAttribute(int *v, hipDeviceAttribute_t a, int) {
    *v = a == hipDeviceAttributeMaxSharedMemoryPerBlock ? 163840 : 256;   // MI355X: 160 KiB, 256 CUs
    return hipSuccess;
}
hipError_t hipMalloc(void **p, size_t n) {
    ++mallocs;
    *p = std::calloc(1, n ? n : 1);
    return *p ? hipSuccess : hipErrorOutOfMemory;
}
hipError_t hipFree(void *p) {
    frees += p != nullptr;
    std::free(p);
    return hipSuccess;
}
hipError_t hipMemcpy(void *d, const void *s, size_t n, hipMemcpyKind) {
    ++copies;
    std::memcpy(d, s, n);
    return hipSuccess;
}
hipError_t hipDeviceSynchronize() { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "host stub"; }
hipError_t hipGetSymbolAddress(void **p, const void *) {
    static char scratch[1 << 16];
    *p = scratch;
    return hipSuccess;
}
hipError_t hipOccupancyMaxActiveBlocksPerMultiprocessor(int *n, const void *, int, size_t) {
    *n = 1;
    return hipSuccess;
}
}

namespace {

template <typename F>
F *entry(void *lib, const char *name) {
    void *p = dlsym(lib, name);
    if (p == nullptr) {
        std::printf("no %s\n", name);
        std::exit(1);
    }
    return reinterpret_cast<F *>(p);
}
#define ENTRY(name) auto *const name = entry<decltype(::name)>(lib, #name)

constexpr int kB = 3, kN1 = 9, kG = 2, kD = 36, kDc = 64, kLdw = 40, kRows = 2 * (kN1 - 1) - 1;
constexpr int64_t kScores = 4 * kB * kN1 * kN1, kTrees = 8 * kB * kG * kRows, kEach = 4 * kB * kG, kVec = 4 * kB;
constexpr int64_t kBf16 = 2 * kB * kN1 * kD, kCodes = kB * kN1 * kDc, kScales = kB * kN1 * kDc / 32, kW = 2 * kD * kLdw;

// Buffers of a call, far apart; a case moves one of them.
struct Buffer {
    const char *name;
    int64_t bytes;
    bool out;
    char *at;
};
// Every pair of an output and another buffer, overlapping at either end (in a
// step of 256 bytes, which keeps every alignment) and side by side.
template <typename CALL>
void pairs(const char *call, std::vector<Buffer> b, CALL &&run) {
    char *base = reinterpret_cast<char *>((uintptr_t)1 << 40);
    for (auto &x : b) x.at = base, base += 1 << 24;
    std::printf("%s none %d\n", call, run(b));
    for (size_t o = 0; o < b.size(); ++o)
        for (size_t i = 0; i < b.size(); ++i) {
            if (i == o || !b[o].out || (b[i].out && i < o)) continue;
            auto with = [&](int64_t shift) {
                auto c = b;
                c[o].at = b[i].at + shift;
                return run(c);
            };
            const int64_t before = (b[o].bytes + 255) / 256 * 256, after = (b[i].bytes + 255) / 256 * 256;
            std::printf("%s %s %s same %d\n", call, b[o].name, b[i].name, with(0));
            std::printf("%s %s %s head %d\n", call, b[o].name, b[i].name, with(after - 256));
            std::printf("%s %s %s tail %d\n", call, b[o].name, b[i].name, with(256 - before));
            std::printf("%s %s %s beside %d\n", call, b[o].name, b[i].name, std::max(with(after), with(-before)));
        }
}
template <typename T>
T *as(const Buffer &b) {
    return reinterpret_cast<T *>(b.at);
}

int aliases(void *lib) {
    ENTRY(crf_plan_create); ENTRY(crf_plan_destroy); ENTRY(crf_tree_workspace); ENTRY(crf_tree_logprobs);
    ENTRY(crf_tree_logprobs_bwd); ENTRY(crf_policy_loss); ENTRY(crf_pack_rows); ENTRY(crf_unpack_rows);
    ENTRY(crf_biaffine_bwd_workspace); ENTRY(crf_biaffine_bwd); ENTRY(crf_biaffine_bwd_packed);
    const int32_t len[kB] = {8, 3, 5};
    crf_plan *p = nullptr;
    if (crf_plan_create(&p, len, kB, kN1, 1, 0) != CRF_OK) return 1;
    int64_t tw = 0, bw = 0;
    crf_tree_workspace(p, &tw);
    crf_biaffine_bwd_workspace(p, kD, 1, &bw);
    pairs("logprobs",
          {{"scores", kScores, false}, {"trees", kTrees, false}, {"counts", kVec, false}, {"logp", kEach, true},
           {"logZ", kVec, true}, {"workspace", tw, true}},
          [&](const std::vector<Buffer> &b) {
              return crf_tree_logprobs(p, as<float>(b[0]), as<int32_t>(b[1]), kG, as<int32_t>(b[2]), as<float>(b[3]),
                                       as<float>(b[4]), b[5].at, tw, nullptr);
          });
    pairs("logprobs_bwd",
          {{"scores", kScores, false}, {"trees", kTrees, false}, {"counts", kVec, false}, {"grad_logp", kEach, false},
           {"grad_scores", kScores, true}},
          [&](const std::vector<Buffer> &b) {
              return crf_tree_logprobs_bwd(p, as<float>(b[0]), as<int32_t>(b[1]), kG, as<int32_t>(b[2]), as<float>(b[3]),
                                           as<float>(b[4]), nullptr);
          });
    pairs("policy",
          {{"scores", kScores, false}, {"trees", kTrees, false}, {"counts", kVec, false}, {"advantages", kEach, false},
           {"old_logp", kEach, false}, {"ref_logp", kEach, false}, {"grad_loss", kVec, false}, {"loss", kVec, true},
           {"logp", kEach, true}, {"grad_scores", kScores, true}, {"workspace", tw, true}},
          [&](const std::vector<Buffer> &b) {
              return crf_policy_loss(p, as<float>(b[0]), as<int32_t>(b[1]), kG, as<int32_t>(b[2]), as<float>(b[3]),
                                     as<float>(b[4]), as<float>(b[5]), 0.2f, 0.2f, 0.1f, as<float>(b[6]), as<float>(b[7]),
                                     as<float>(b[8]), as<float>(b[9]), b[10].at, tw, nullptr);
          });
    pairs("pack", {{"x", kBf16, false}, {"codes", kCodes, true}, {"scales", kScales, true}},
          [&](const std::vector<Buffer> &b) {
              return crf_pack_rows(p, as<uint16_t>(b[0]), kD, as<uint8_t>(b[1]), as<uint8_t>(b[2]), nullptr);
          });
    pairs("unpack", {{"codes", kCodes, false}, {"scales", kScales, false}, {"x", kBf16, true}},
          [&](const std::vector<Buffer> &b) {
              return crf_unpack_rows(p, as<uint8_t>(b[0]), as<uint8_t>(b[1]), kD, as<uint16_t>(b[2]), nullptr);
          });
    pairs("bwd",
          {{"rl", kBf16, false}, {"rr", kBf16, false}, {"w", kW, false}, {"grad_scores", kScores, false},
           {"grad_rl", kBf16, true}, {"grad_rr", kBf16, true}, {"grad_w", 2 * kW, true}, {"workspace", bw, true}},
          [&](const std::vector<Buffer> &b) {
              return crf_biaffine_bwd(p, as<uint16_t>(b[0]), as<uint16_t>(b[1]), as<uint16_t>(b[2]), kD, kLdw, 1,
                                      as<float>(b[3]), as<uint16_t>(b[4]), as<uint16_t>(b[5]), as<float>(b[6]), b[7].at, bw,
                                      nullptr);
          });
    pairs("bwd_packed",
          {{"rl_codes", kCodes, false}, {"rl_scales", kScales, false}, {"rr_codes", kCodes, false},
           {"rr_scales", kScales, false}, {"w", kW, false}, {"grad_scores", kScores, false}, {"grad_rl", kBf16, true},
           {"grad_rr", kBf16, true}, {"grad_w", 2 * kW, true}, {"workspace", bw, true}},
          [&](const std::vector<Buffer> &b) {
              return crf_biaffine_bwd_packed(p, as<uint8_t>(b[0]), as<uint8_t>(b[1]), as<uint8_t>(b[2]), as<uint8_t>(b[3]),
                                             as<uint16_t>(b[4]), kD, kLdw, 1, as<float>(b[5]), as<uint16_t>(b[6]),
                                             as<uint16_t>(b[7]), as<float>(b[8]), b[9].at, bw, nullptr);
          });
    crf_plan_destroy(p);
    return 0;
}

// Two threads whose first calls of the scorer's backward pass meet.
int attributes(void *lib) {
    ENTRY(crf_plan_create); ENTRY(crf_plan_destroy); ENTRY(crf_biaffine_bwd_workspace); ENTRY(crf_biaffine_bwd);
    const int32_t len[kB] = {8, 3, 100};
    constexpr int d = 500, ldw = 504, n1 = 101;
    crf_plan *p[2] = {nullptr, nullptr};
    for (auto &x : p)
        if (crf_plan_create(&x, len, kB, n1, 1, 0) != CRF_OK) return 1;
    int64_t bytes = 0;
    crf_biaffine_bwd_workspace(p[0], d, 1, &bytes);
    ready.clear();
    launched.clear();
    slow_attributes = watch_attributes = true;
    int rc[2] = {0, 0};
    auto call = [&](int t) {
        auto at = [&](int k) { return reinterpret_cast<char *>(((uintptr_t)1 << 40) + ((uintptr_t)(16 * t + k) << 28)); };
        rc[t] = crf_biaffine_bwd(p[t], (uint16_t *)at(0), (uint16_t *)at(1), (uint16_t *)at(2), d, ldw, 1, (float *)at(3),
                                 (uint16_t *)at(4), (uint16_t *)at(5), (float *)at(6), at(7), bytes, nullptr);
    };
    std::thread a(call, 0), b([&]() {
        std::this_thread::sleep_for(std::chrono::milliseconds(5));   // the first thread is at its attributes
        call(1);
    });
    a.join();
    b.join();
    for (const std::string &x : early) std::printf("EARLY %s\n", x.c_str());
    std::printf("launches %d status %d %d\n", (int)launched.size(), rc[0], rc[1]);
    for (auto *x : p) crf_plan_destroy(x);
    return 0;
}

int memory(void *lib, const std::vector<int32_t> &len) {
    ENTRY(crf_plan_create); ENTRY(crf_plan_destroy); ENTRY(crf_last_error);
    int last = -1, times = 0;
    mallocs = frees = 0;
    auto tell = [&]() {
        if (times > 0) std::printf("status %d times %d\n", last, times);
    };
    for (int64_t k = 0; last != CRF_OK; ++k) {
        crf_plan *p = nullptr;
        news_left = k;
        const int rc = crf_plan_create(&p, len.data(), (int32_t)len.size(), *std::max_element(len.begin(), len.end()) + 1, 1, 0);
        news_left = -1;
        if (rc != CRF_OK && (p != nullptr || crf_last_error()[0] == 0)) return 1;
        if (rc == CRF_OK) crf_plan_destroy(p);
        if (rc != last) tell(), times = 0;
        last = rc;
        ++times;
    }
    tell();
    std::printf("left %d\n", mallocs - frees);
    return 0;
}

int creation(void *lib, const std::vector<int32_t> &len) {
    ENTRY(crf_plan_create); ENTRY(crf_plan_destroy);
    crf_plan *p = nullptr;
    mallocs = copies = 0;
    if (crf_plan_create(&p, len.data(), (int32_t)len.size(), *std::max_element(len.begin(), len.end()) + 1, 1, 0) != CRF_OK)
        return 1;
    std::printf("mallocs %d copies %d\n", mallocs, copies);
    crf_plan_destroy(p);
    return 0;
}

int launches(void *lib, const std::string &call, int flags, const std::vector<int32_t> &len) {
    ENTRY(crf_plan_create); ENTRY(crf_plan_destroy); ENTRY(crf_tree_workspace); ENTRY(crf_tree_logprobs);
    ENTRY(crf_tree_logprobs_bwd); ENTRY(crf_policy_loss); ENTRY(crf_inside_fwd_bwd);
    crf_plan *p = nullptr;
    if (crf_plan_create(&p, len.data(), (int32_t)len.size(), *std::max_element(len.begin(), len.end()) + 1, 1, flags) != CRF_OK)
        return 1;
    int64_t tw = 0;
    crf_tree_workspace(p, &tw);
    launched.clear();
    auto f = [](int k) { return reinterpret_cast<float *>((uintptr_t)(k + 1) << 40); };
    const int32_t *trees = reinterpret_cast<int32_t *>(f(0));
    int rc = -1;
    if (call == "logprobs") rc = crf_tree_logprobs(p, f(1), trees, 2, nullptr, f(2), nullptr, workspace, tw, nullptr);
    if (call == "logprobs_bwd") rc = crf_tree_logprobs_bwd(p, f(1), trees, 2, nullptr, f(2), f(3), nullptr);
    if (call == "policy")
        rc = crf_policy_loss(p, f(1), trees, 2, nullptr, f(2), f(3), nullptr, 0.2f, 0.2f, 0.f, nullptr, f(4), f(5), f(6),
                             workspace, tw, nullptr);
    if (call == "inside") rc = crf_inside_fwd_bwd(p, f(1), nullptr, f(2), f(3), nullptr);
    for (const std::string &x : launched) std::printf("K %s\n", x.c_str());
    for (const std::string &x : marked) std::printf("%s\n", x.c_str());
    crf_plan_destroy(p);
    return rc;
}

}  // namespace

int main(int argc, char **argv) {
    if (argc < 3) return 2;
    void *lib = dlopen(argv[2], RTLD_NOW);
    if (lib == nullptr) {
        std::printf("%s\n", dlerror());
        return 1;
    }
    const std::string mode = argv[1];
    if (mode == "alias") return aliases(lib);
    if (mode == "attributes") return attributes(lib);
    if ((mode == "creation" || mode == "memory") && argc > 3) {
        std::vector<int32_t> len;
        for (int k = 3; k < argc; ++k) len.push_back(std::atoi(argv[k]));
        return mode == "memory" ? memory(lib, len) : creation(lib, len);
    }
    if (mode == "launches" && argc > 5) {
        std::vector<int32_t> len;
        for (int k = 5; k < argc; ++k) len.push_back(std::atoi(argv[k]));
        return launches(lib, argv[3], std::atoi(argv[4]), len);
    }
    return 2;
}
