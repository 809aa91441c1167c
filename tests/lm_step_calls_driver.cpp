// Calls of the operators around a language model's layers without a GPU, as lm_calls_driver.cpp makes those of its own, with its stand-in for the runtime.
//   lm_step_calls_driver libnetmax.so < calls
// A call is a line: embed, embed_grad, norm, norm_grad, grad_norm or clip, then name=number for members of its shape and its arguments; what is not named is 0.  A span is named by its
// address, with .ld and .s behind the name for its distances; gradients are numbered: g0, out0, rows0 ...
#define main lm_calls_main
#include "lm_calls_driver.cpp"
#undef main

#include <vector>

int main(int argc, char **argv)
{
    void *lib = argc == 2 ? dlopen(argv[1], RTLD_NOW) : nullptr;
    if (!lib) {
        fprintf(stderr, "%s\n", argc == 2 ? dlerror() : "usage: lm_step_calls_driver libnetmax.so < calls");
        return 2;
    }
#define ENTRY(name) const auto name##_ = reinterpret_cast<decltype(&name)>(dlsym(lib, #name))
    ENTRY(netmax_embed); ENTRY(netmax_embed_grad); ENTRY(netmax_embed_grad_workspace); ENTRY(netmax_block_norm); ENTRY(netmax_block_norm_grad); ENTRY(netmax_block_norm_grad_workspace);
    ENTRY(netmax_grad_norm); ENTRY(netmax_grad_norm_workspace); ENTRY(netmax_clip_grads); ENTRY(netmax_last_error);
#undef ENTRY
    for (std::string line; std::getline(std::cin, line);) {
        std::istringstream in(line);
        std::string op;
        in >> op;
        std::map<std::string, double> v;
        for (std::string word; in >> word;) v[word.substr(0, word.find('='))] = std::stod(word.substr(word.find('=') + 1));
        const auto n = [&](const std::string &name) { return (int64_t)v[name]; };
        const auto f = [&](const char *name) { return (float)v[name]; };
        const auto p = [&](const std::string &name) { return reinterpret_cast<float *>((uintptr_t)v[name]); };
        const auto span = [&](const std::string &name) { return netmax_span{p(name), n(name + ".ld"), n(name + ".s")}; };
        g_out.str("");
        int rc = -100;
        if (op == "kernels")
            for (const auto &k : g_names) g_out << ' ' << k.second << "@0";
        if (op == "embed" || op == "embed_grad") {
            const netmax_embed_shape s{n("batch"), n("tokens"), n("vocab"), n("width"), (int32_t)n("dtype"), (int32_t)n("accumulate"), 1.0f, n("s_ids"), n("ldt"), n("st"), n("ldy"), n("sy")};
            const int32_t *ids = reinterpret_cast<int32_t *>((uintptr_t)v["ids"]);
            rc = op == "embed" ? netmax_embed_(&s, ids, p("table"), p("y"), nullptr) : netmax_embed_grad_(&s, ids, p("y"), p("table"), p("work"), netmax_embed_grad_workspace_(&s), nullptr);
        } else if (op == "norm" || op == "norm_grad") {
            const netmax_block_norm_shape s{n("batch"), n("rows"), n("width"), (int32_t)n("dtype"), (int32_t)n("norm"), (int32_t)n("gate_act"), (int32_t)n("gate_rows"), (int32_t)n("post"), (int32_t)n("pre"),
                                            f("x_scale"), f("f_scale"), f("eps")};
            const netmax_block_norm_data d{span("x"), span("f"), span("gate"), span("post_gain"), span("post_bias"), span("pre_gain"), span("pre_bias"), span("h"), span("y")};
            const netmax_block_norm_grads g{span("dy"), span("dh"), span("dx"), span("df"), span("dgate"), span("dpost_gain"), span("dpost_bias"), span("dpre_gain"), span("dpre_bias")};
            rc = op == "norm" ? netmax_block_norm_(&s, &d, nullptr) : netmax_block_norm_grad_(&s, &d, &g, p("work"), netmax_block_norm_grad_workspace_(&s, &d, &g), nullptr);
        } else if (op == "grad_norm" || op == "clip") {
            std::vector<netmax_gradient> g((size_t)n("n"));
            for (size_t k = 0; k < g.size(); ++k) {
                const std::string i = std::to_string(k);
                g[k] = netmax_gradient{p("g" + i), p("out" + i), n("rows" + i), n("cols" + i), n("ldg" + i), n("sg" + i), n("ldo" + i), n("so" + i), (int32_t)n("dtype" + i)};
            }
            const int64_t bytes = netmax_grad_norm_workspace_(n("batch"), n("n"), g.data());
            rc = op == "clip" ? netmax_clip_grads_(n("batch"), n("n"), g.data(), 1.0f, p("norm"), p("work"), bytes, nullptr)
                              : netmax_grad_norm_(n("batch"), n("n"), g.data(), p("norm"), p("work"), bytes, nullptr);
        }
        printf("%d|%s|%s\n", rc, rc == NETMAX_OK ? "" : netmax_last_error_(nullptr), g_out.str().c_str());
    }
    return 0;
}
