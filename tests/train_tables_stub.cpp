// The fine-tuning operators' tables of a plan, on the host: the plan built as
// in plan_host_stub.cpp, printed as
//   H B n1 n_posts n_long_posts n_tree_recs tree_cells cells
//   P square compact rest id   one line a place of a block (rest: the record's n - i)
//   F first last               one line a block
//   T b n row rows             one line a stripe
// Arguments: a file of sentence lengths.
#define main plan_main
#include "plan_host_stub.cpp"
#undef main

int main(int argc, char **argv) {
    if (argc < 2) return 2;
    std::vector<int32_t> len;
    FILE *f = std::fopen(argv[1], "r");
    if (f == nullptr) return 2;
    for (int v; std::fscanf(f, "%d", &v) == 1;) len.push_back(v);
    std::fclose(f);
    crf_plan *p = nullptr;
    const int32_t n1 = *std::max_element(len.begin(), len.end()) + 1;
    if (crf_plan_create(&p, len.data(), (int32_t)len.size(), n1, 1, 0) != CRF_OK) {
        std::printf("%s\n", crf_last_error());
        return 1;
    }
    const crf::KernelPlan &k = p->kp;
    std::printf("H %d %d %d %d %d %d %lld\n", k.B, k.n1, k.n_posts, k.n_long_posts, k.n_tree_recs, k.tree_cells,
                (long long)p->cells);
    const int slots = k.n_posts * crf::kBiaRows;
    for (int q = 0; q < k.n_posts; ++q) {
        const int32_t *rec = k.posts + (size_t)q * crf::kPostRec;
        for (int r = 0; r < crf::kBiaRows; ++r)
            std::printf("P %lld %lld %d %d\n", (long long)k.post_cells[q * crf::kBiaRows + r],
                        (long long)k.post_cells[slots + q * crf::kBiaRows + r], rec[crf::kBiaRows + r], rec[r]);
        std::printf("F %d %d\n", rec[2 * crf::kBiaRows], rec[2 * crf::kBiaRows + 1]);
    }
    for (int q = 0; q < k.n_tree_recs; ++q) {
        const int32_t *rec = k.tree_recs + 4 * q;
        std::printf("T %d %d %d %d\n", rec[0], rec[1], rec[2], rec[3]);
    }
    crf_plan_destroy(p);
    return 0;
}
