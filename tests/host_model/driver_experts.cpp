// Calls of include/mxfp8_experts.h on the CPU execution model (tests/host_model/wavesim.h). A line of the case file is
//   <entry point> <argument> ...
// with an argument for each of the entry point's but the stream:
//   <number>            as it is
//   null
//   in:<file>           a buffer of exactly the file's bytes, which the call must leave unchanged
//   out:<file>:<bytes>  a buffer of that many bytes 0xA5, written to the file after the call
//   off:<n>:<argument>  a buffer as in: or out:, n bytes (of it) further on
// Buffers are heap blocks of their exact size (AddressSanitizer guards their ends), 16-byte aligned. Prints the status of each call.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <fstream>
#include <sstream>
#include <string>
#include <vector>

#include "../../include/mxfp8_experts.h"
#include "wavesim.h"

extern "C" const char *__asan_default_options() { return "detect_leaks=0:detect_stack_use_after_return=0"; }

namespace {
struct Buf {
    uint8_t *p;
    size_t n;
    std::vector<uint8_t> copy;
    std::string to;  // outputs: their file
};

uint8_t *block(size_t n)
{
    void *p = nullptr;
    if (posix_memalign(&p, 16, n ? n : 1) != 0)
        exit(2);
    return static_cast<uint8_t *>(p);
}

int64_t argument(const std::string &a, std::vector<Buf> &buffers)
{
    if (a == "null")
        return 0;
    if (a.rfind("off:", 0) == 0) {
        const size_t colon = a.find(':', 4);
        return argument(a.substr(colon + 1), buffers) + atoll(a.substr(4, colon - 4).c_str());
    }
    if (a.rfind("in:", 0) == 0) {
        std::ifstream f(a.substr(3), std::ios::binary);
        if (!f) {
            fprintf(stderr, "cannot open %s\n", a.c_str());
            exit(2);
        }
        std::vector<uint8_t> bytes((std::istreambuf_iterator<char>(f)), std::istreambuf_iterator<char>());
        uint8_t *p = block(bytes.size());
        memcpy(p, bytes.data(), bytes.size());
        buffers.push_back({p, bytes.size(), bytes, ""});
        return (int64_t)p;
    }
    if (a.rfind("out:", 0) == 0) {
        const size_t colon = a.rfind(':');
        const size_t n = (size_t)atoll(a.substr(colon + 1).c_str());
        uint8_t *p = block(n);
        memset(p, 0xA5, n);
        buffers.push_back({p, n, {}, a.substr(4, colon - 4)});
        return (int64_t)p;
    }
    return atoll(a.c_str());
}
}  // namespace

int main(int argc, char **argv)
{
    std::ifstream in(argc > 1 ? argv[1] : "");
    std::string line;
    while (std::getline(in, line)) {
        std::istringstream ls(line);
        std::string name, a;
        if (!(ls >> name))
            continue;
        std::vector<Buf> buffers;
        std::vector<int64_t> v;
        while (ls >> a)
            v.push_back(argument(a, buffers));
        auto p = [&](size_t i) { return (uint8_t *)v.at(i); };
        auto w = [&](size_t i) { return (int32_t *)v.at(i); };
        int st = -1;
        if (name == "sort")
            st = mxfp8_expert_sort(p(0), (mxfp8_index)v.at(1), v.at(2), (int32_t)v.at(3), (int32_t)v.at(4), v.at(5), w(6), w(7), w(8), p(9), nullptr);
        else if (name == "quantize")
            st = mxfp8_expert_quantize_ex(p(0), (mxfp8_dtype)v.at(1), v.at(2), v.at(3), v.at(4), w(5), (int32_t)v.at(6), (float *)p(7), w(8),
                                          (int32_t)v.at(9), v.at(10), (mxfp8_axis)v.at(11), p(12), p(13), p(14), p(15), (mxfp8_scale_layout)v.at(16), nullptr);
        else if (name == "combine")
            st = mxfp8_expert_combine(p(0), (mxfp8_dtype)v.at(1), v.at(2), v.at(3), v.at(4), w(5), (float *)p(6), v.at(7), (int32_t)v.at(8), p(9),
                                      (mxfp8_dtype)v.at(10), v.at(11), nullptr);
        else if (name == "weight_grad")
            st = mxfp8_expert_weight_grad(p(0), (mxfp8_dtype)v.at(1), v.at(2), p(3), (mxfp8_dtype)v.at(4), v.at(5), v.at(6), v.at(7), w(8), v.at(9),
                                          (int32_t)v.at(10), (float *)p(11), nullptr);
        else if (name == "gemv")
            st = mxfp8_fp4_gemv_ex(p(0), v.at(1), p(2), p(3), v.at(4), v.at(5), v.at(6), p(7), (mxfp8_dtype)v.at(8), v.at(9), (mxfp8_scale_layout)v.at(10), nullptr);
        else if (name == "gemv_grouped")
            st = mxfp8_fp4_gemv_grouped_ex(p(0), v.at(1), v.at(2), w(3), (int32_t)v.at(4), p(5), p(6), w(7), (int32_t)v.at(8), v.at(9), v.at(10), v.at(11),
                                           p(12), (mxfp8_dtype)v.at(13), v.at(14), (mxfp8_scale_layout)v.at(15), nullptr);
        else
            return 2;
        printf("status %d workgroups %u\n", st, wavesim::g.call_launches.empty() ? 0 : wavesim::g.call_launches.back().first);
        fflush(stdout);
        for (Buf &b : buffers) {
            if (b.to.empty()) {
                if (b.n && memcmp(b.p, b.copy.data(), b.n) != 0) {
                    fprintf(stderr, "%s: the call modified an input\n", name.c_str());
                    return 4;
                }
            } else {
                std::ofstream(b.to, std::ios::binary).write((const char *)b.p, (std::streamsize)b.n);
            }
            free(b.p);
        }
    }
    return 0;
}
