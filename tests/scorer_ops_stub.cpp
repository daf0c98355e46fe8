// Layer norm, the width bias and the orthogonalised update of the built library
// on launch_host_stub.cpp's HIP runtime of host memory.  Modes:
//   alias LIB                    "call name ... status" of calls whose buffers overlap or touch
//   grids LIB D LABELS LENGTHS...   "L name grid(x y z) threads lds" of each launch of layer
//                                norm and of the width bias
//   update LIB COUNT ROWS COLS   the same of the orthogonalised update
//   products LIB SIDES COUNTS    "T kind tiles k" of each product in tiles of 64 x tiles that
//                                the update launches for matrices of up to SIDES x 64 rows and
//                                columns, 1 to COUNTS of them
//   steps LIB STEPS A B C ...    the status of the update with each set of that many steps' coefficients
//   eps LIB EPS ...              the statuses of layer norm and of its backward pass with each
//   biased LIB                   "A name" of each scorer kernel whose attribute a plan's creation sets, then
//                                of two threads' first calls of the scorer with a bias "EARLY name" of each
//                                kernel launched before its attribute was set, and "launches N"
#define main launch_main
#define hipLaunchKernel plain_hipLaunchKernel
#include "launch_host_stub.cpp"
#undef hipLaunchKernel
#undef main

namespace {
std::vector<std::string> shapes;
std::set<std::string> products;
// The head of what a product's kernel is passed (crf_ortho.hip).
struct ProductHead {
    const void *left, *right, *add, *out, *out_t;
    int k, stride, t_stride, across;
};
}

extern "C" hipError_t hipLaunchKernel(const void *f, dim3 g, dim3 b, void **args, size_t lds, hipStream_t) {
    std::lock_guard<std::mutex> lock(mu);
    if (watch_attributes && lds > 65536 && ready.count(f) == 0) early.push_back(names[f]);
    std::string name = names[f];
    const size_t tile = name.find("ortho_tile_kernel<");
    if (tile != std::string::npos) {   // (kind and tiles are its template's arguments, the kind perhaps with its type)
        std::string of = name.substr(tile + 18, name.find('>', tile) - tile - 18);
        const size_t kind = of.rfind(')', of.find(','));
        if (kind != std::string::npos) of = of.substr(kind + 1);
        of.erase(of.find(','), 1);
        products.insert("T " + of + " " + std::to_string(static_cast<const ProductHead *>(args[0])->k));
    }
    const size_t end = name.find('('), start = name.find("(anonymous namespace)::");
    name = start != std::string::npos && start < name.find("_kernel") ? name.substr(start + 23) : name.substr(0, end);
    name = name.substr(0, name.find_first_of("(<"));
    shapes.push_back("L " + name + " " + std::to_string(g.x) + " " + std::to_string(g.y) + " " + std::to_string(g.z) + " " +
                     std::to_string(b.x * b.y * b.z) + " " + std::to_string(lds));
    return hipSuccess;
}

namespace {

const float kSteps[2][3] = {{3.4445f, -4.7750f, 2.0315f}, {1.5f, -0.5f, 0.f}};

int op_aliases(void *lib) {
    ENTRY(crf_plan_create); ENTRY(crf_plan_destroy); ENTRY(crf_layer_norm); ENTRY(crf_layer_norm_bwd);
    ENTRY(crf_layer_norm_bwd_workspace); ENTRY(crf_width_bias); ENTRY(crf_width_bias_bwd);
    ENTRY(crf_width_bias_bwd_workspace); ENTRY(crf_orthogonalize); ENTRY(crf_orthogonalize_workspace); ENTRY(crf_muon_step);
    ENTRY(crf_biaffine_scores_biased);
    const int32_t len[kB] = {8, 3, 5};
    constexpr int64_t rows = (int64_t)kB * kN1 * kD, vec = 4 * kD, K = 5, L = 3;
    crf_plan *p = nullptr;
    if (crf_plan_create(&p, len, kB, kN1, 1, 0) != CRF_OK) return 1;
    int64_t nw = 0, ww = 0, ow = 0;
    crf_layer_norm_bwd_workspace(p, kD, &nw);
    crf_width_bias_bwd_workspace(p, (int)L, &ww);
    crf_orthogonalize_workspace(2, 20, 30, &ow);
    pairs("norm", {{"x", 4 * rows, false}, {"gamma", vec, false}, {"beta", vec, false}, {"y", 2 * rows, true}},
          [&](const std::vector<Buffer> &b) {
              return crf_layer_norm(p, b[0].at, CRF_F32, kD, as<float>(b[1]), as<float>(b[2]), 1e-5f, as<uint16_t>(b[3]),
                                    nullptr);
          });
    pairs("norm_bwd",
          {{"x", 4 * rows, false}, {"gamma", vec, false}, {"grad_y", 2 * rows, false}, {"grad_x", 4 * rows, true},
           {"grad_gamma", vec, true}, {"grad_beta", vec, true}, {"workspace", nw, true}},
          [&](const std::vector<Buffer> &b) {
              return crf_layer_norm_bwd(p, b[0].at, CRF_F32, kD, as<float>(b[1]), as<uint16_t>(b[2]), 1e-5f, b[3].at,
                                        as<float>(b[4]), as<float>(b[5]), b[6].at, nw, nullptr);
          });
    pairs("width",
          {{"scores", L * kScores, false}, {"table", 4 * K * L, false}, {"buckets", 4 * kN1, false}, {"out", L * kScores, true}},
          [&](const std::vector<Buffer> &b) {
              return crf_width_bias(p, as<float>(b[0]), (int)L, as<float>(b[1]), as<int32_t>(b[2]), (int)K, as<float>(b[3]),
                                    nullptr);
          });
    pairs("width_bwd",
          {{"grad_out", L * kScores, false}, {"buckets", 4 * kN1, false}, {"grad_scores", L * kScores, true},
           {"grad_table", 4 * K * L, true}, {"workspace", ww, true}},
          [&](const std::vector<Buffer> &b) {
              return crf_width_bias_bwd(p, as<float>(b[0]), (int)L, as<int32_t>(b[1]), (int)K, as<float>(b[2]), as<float>(b[3]),
                                        b[4].at, ww, nullptr);
          });
    pairs("scorer",
          {{"rl", kBf16, false}, {"rr", kBf16, false}, {"w", kW, false}, {"table", 4 * K, false}, {"buckets", 4 * kN1, false},
           {"scores", kScores, true}},
          [&](const std::vector<Buffer> &b) {
              return crf_biaffine_scores_biased(p, as<uint16_t>(b[0]), as<uint16_t>(b[1]), as<uint16_t>(b[2]), kD, kLdw, 1,
                                                as<float>(b[3]), as<int32_t>(b[4]), (int)K, as<float>(b[5]), nullptr);
          });
    constexpr int64_t all = 4 * 2 * 20 * 32;
    pairs("ortho", {{"x", all, false}, {"out", all, true}, {"workspace", ow, true}}, [&](const std::vector<Buffer> &b) {
        return crf_orthogonalize(as<float>(b[0]), 2, 20, 30, 32, kSteps[0], 2, 1e-7f, as<float>(b[1]), b[2].at, ow, nullptr);
    });
    pairs("muon",
          {{"w", all, false}, {"grad", all, false}, {"momentum", all, false}, {"w_out", all, true}, {"momentum_out", all, true},
           {"workspace", ow, true}},
          [&](const std::vector<Buffer> &b) {
              return crf_muon_step(as<float>(b[0]), as<float>(b[1]), as<float>(b[2]), 2, 20, 30, 32, 0.9f, 1, 0.1f, 0.01f,
                                   kSteps[0], 2, 1e-7f, as<float>(b[3]), as<float>(b[4]), b[5].at, ow, nullptr);
          });
    crf_plan_destroy(p);
    return 0;
}

int grids(void *lib, int d, int labels, const std::vector<int32_t> &len) {
    ENTRY(crf_plan_create); ENTRY(crf_plan_destroy); ENTRY(crf_layer_norm); ENTRY(crf_layer_norm_bwd);
    ENTRY(crf_layer_norm_bwd_workspace); ENTRY(crf_width_bias); ENTRY(crf_width_bias_bwd);
    ENTRY(crf_width_bias_bwd_workspace);
    crf_plan *p = nullptr;
    if (crf_plan_create(&p, len.data(), (int32_t)len.size(), *std::max_element(len.begin(), len.end()) + 1, 1, 0) != CRF_OK)
        return 1;
    int64_t nw = 0, ww = 0;
    crf_layer_norm_bwd_workspace(p, d, &nw);
    crf_width_bias_bwd_workspace(p, labels, &ww);
    auto f = [](int k) { return reinterpret_cast<float *>((uintptr_t)(k + 1) << 44); };
    shapes.clear();
    for (int type : {CRF_BF16, CRF_F32}) {
        if (crf_layer_norm(p, f(0), type, d, nullptr, nullptr, 1e-5f, (uint16_t *)f(1), nullptr) != CRF_OK) return 2;
        if (crf_layer_norm_bwd(p, f(0), type, d, f(1), (uint16_t *)f(2), 1e-5f, f(3), f(4), f(5), f(6), nw, nullptr) != CRF_OK)
            return 3;
    }
    if (crf_width_bias(p, f(0), labels, f(1), (int32_t *)f(2), 1024, f(3), nullptr) != CRF_OK) return 4;
    if (crf_width_bias_bwd(p, f(0), labels, (int32_t *)f(2), 1024, f(3), f(4), f(5), ww, nullptr) != CRF_OK) return 5;
    for (const std::string &s : shapes) std::printf("%s\n", s.c_str());
    crf_plan_destroy(p);
    return 0;
}

int update(void *lib, int count, int rows, int cols) {
    ENTRY(crf_muon_step); ENTRY(crf_orthogonalize); ENTRY(crf_orthogonalize_workspace);
    int64_t ow = 0;
    if (crf_orthogonalize_workspace(count, rows, cols, &ow) != CRF_OK) return 1;
    auto f = [](int k) { return reinterpret_cast<float *>((uintptr_t)(k + 1) << 44); };
    shapes.clear();
    if (crf_orthogonalize(f(0), count, rows, cols, cols, kSteps[0], 2, 1e-7f, f(1), f(2), ow, nullptr) != CRF_OK) return 2;
    if (crf_muon_step(f(0), f(1), f(2), count, rows, cols, cols, 0.9f, 1, 0.1f, 0.01f, kSteps[0], 2, 1e-7f, f(0), f(2), f(3), ow,
                      nullptr) != CRF_OK)
        return 3;
    return 0;
}

int tile_products(void *lib, int sides, int counts) {
    for (int p = 1; p <= sides; ++p)
        for (int q = p; q <= sides; ++q)
            for (int count = 1; count <= counts; ++count) {
                // (a side's last rows of padding may be all there, or none)
                const int rc = (count & 1) != 0 ? update(lib, count, 64 * p, 64 * q) : update(lib, count, 64 * q - 7, 64 * p - 9);
                if (rc != 0) return rc;
            }
    for (const std::string &s : products) std::printf("%s\n", s.c_str());
    return 0;
}

int steps(void *lib, int count, const std::vector<float> &all) {
    ENTRY(crf_orthogonalize);
    auto f = [](int k) { return reinterpret_cast<float *>((uintptr_t)(k + 1) << 44); };
    for (size_t k = 0; k + 3 * count <= all.size(); k += 3 * count)
        std::printf("%d\n", crf_orthogonalize(f(0), 1, 8, 8, 8, &all[k], count, 1e-7f, f(1), f(2), 1 << 20, nullptr));
    return 0;
}

int biased(void *lib) {
    ENTRY(crf_plan_create); ENTRY(crf_plan_destroy); ENTRY(crf_biaffine_scores_biased);
    const int32_t len[kB] = {8, 3, 100};
    crf_plan *p[2] = {nullptr, nullptr};
    for (auto &x : p)
        if (crf_plan_create(&x, len, kB, 101, 1, 0) != CRF_OK) return 1;
    for (const void *f : ready)
        if (names[f].find("biaffine") != std::string::npos) std::printf("A %s\n", names[f].c_str());
    shapes.clear();
    slow_attributes = watch_attributes = true;
    int rc[2] = {0, 0};
    auto call = [&](int t) {
        auto at = [&](int k) { return reinterpret_cast<char *>(((uintptr_t)1 << 40) + ((uintptr_t)(16 * t + k) << 28)); };
        rc[t] = crf_biaffine_scores_biased(p[t], (uint16_t *)at(0), (uint16_t *)at(1), (uint16_t *)at(2), 500, 504, 1,
                                           (float *)at(3), (int32_t *)at(4), 4, (float *)at(5), nullptr);
    };
    std::thread a(call, 0), b([&]() {
        std::this_thread::sleep_for(std::chrono::milliseconds(5));   // the first thread is at its attributes
        call(1);
    });
    a.join();
    b.join();
    for (const std::string &x : early) std::printf("EARLY %s\n", x.c_str());
    std::printf("launches %d status %d %d\n", (int)shapes.size(), rc[0], rc[1]);
    for (auto *x : p) crf_plan_destroy(x);
    return 0;
}

int norm_eps(void *lib, const std::vector<float> &all) {
    ENTRY(crf_plan_create); ENTRY(crf_plan_destroy); ENTRY(crf_layer_norm); ENTRY(crf_layer_norm_bwd);
    ENTRY(crf_layer_norm_bwd_workspace);
    const int32_t len[kB] = {8, 3, 5};
    crf_plan *p = nullptr;
    if (crf_plan_create(&p, len, kB, kN1, 1, 0) != CRF_OK) return 1;
    int64_t nw = 0;
    crf_layer_norm_bwd_workspace(p, kD, &nw);
    auto f = [](int k) { return reinterpret_cast<float *>((uintptr_t)(k + 1) << 44); };
    for (const float eps : all)
        std::printf("%d %d\n", crf_layer_norm(p, f(0), CRF_F32, kD, nullptr, nullptr, eps, (uint16_t *)f(1), nullptr),
                    crf_layer_norm_bwd(p, f(0), CRF_F32, kD, nullptr, (uint16_t *)f(1), eps, f(2), f(3), f(4), f(5), nw,
                                       nullptr));
    crf_plan_destroy(p);
    return 0;
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
    if (mode == "alias") return op_aliases(lib);
    if (mode == "biased") return biased(lib);
    std::vector<float> all;
    for (int k = 3; k < argc; ++k) all.push_back(std::strtof(argv[k], nullptr));
    if (mode == "steps" && argc > 6) return steps(lib, std::atoi(argv[3]), std::vector<float>(all.begin() + 1, all.end()));
    if (mode == "eps" && argc > 3) return norm_eps(lib, all);
    std::vector<int> v;
    for (int k = 3; k < argc; ++k) v.push_back(std::atoi(argv[k]));
    if (mode == "grids" && v.size() > 2) return grids(lib, v[0], v[1], std::vector<int32_t>(v.begin() + 2, v.end()));
    if (mode == "update" && v.size() == 3) {
        const int rc = update(lib, v[0], v[1], v[2]);
        for (const std::string &s : shapes) std::printf("%s\n", s.c_str());
        return rc;
    }
    if (mode == "products" && v.size() == 2) return tile_products(lib, v[0], v[1]);
    return 2;
}
