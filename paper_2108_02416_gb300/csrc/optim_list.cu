// Lists of tensors for the norm, clipping and AdamW: argument checks and the
// launch tables.  Host only.
#include <math.h>

#include <algorithm>
#include <new>

#include "optim.cuh"

using namespace aspis;

namespace {

constexpr int64_t kMostElements = (int64_t)1 << 38;      // keeps units within 31 bits

bool known(int type) { return type == ASPIS_F32 || type == ASPIS_BF16 || type == ASPIS_F16; }

aspis_status check_array(const void *p, int64_t numel, int type)
{
    if (!known(type) || numel < 0 || (numel > 0 && !p)) return ASPIS_E_INVAL;
    if (numel > kMostElements) return ASPIS_E_RANGE;
    if (numel > 0 && (uintptr_t)p % (uintptr_t)type_bytes(type) != 0) return ASPIS_E_ALIGN;
    return ASPIS_OK;
}

// Ranges of bytes and what happens to them: whether some range that is written
// meets another.
struct Ranges {
    struct Range {
        uintptr_t begin, end;
        bool written;
    };
    std::vector<Range> all;

    void add(const void *p, int64_t bytes, bool written)
    {
        if (bytes > 0) all.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, written});
    }
    bool apart()
    {
        std::sort(all.begin(), all.end(), [](const Range &a, const Range &b) { return a.begin < b.begin; });
        uintptr_t end = 0, written_end = 0;       // of the ranges so far, and of the written ones
        for (const Range &r : all) {
            if (r.begin < written_end || (r.written && r.begin < end)) return false;
            end = std::max(end, r.end);
            if (r.written) written_end = std::max(written_end, r.end);
        }
        return true;
    }
};

// up to 7 elements before the first aligned group shift a tensor's units
uint32_t units_of(int64_t numel, int unit) { return numel ? (uint32_t)((numel + 7 + unit - 1) / unit) : 1; }

// Appends tensors to tables of at most N entries (and 2^31 units).
template <class T, class E, int N>
void append(std::vector<std::unique_ptr<T>> &tables, E e, uint32_t units, int64_t index)
{
    if (tables.empty() || tables.back()->n == N || (uint64_t)tables.back()->units + units > (1u << 31)) {
        tables.push_back(std::make_unique<T>());
        tables.back()->n = 0;
        tables.back()->units = 0;
        tables.back()->first = (int32_t)index;
        tables.back()->last = 0;
    }
    T &t = *tables.back();
    e.begin = t.units;
    t.units += units;
    e.end = t.units;
    t.e[t.n++] = e;
}

template <class T>
void finish(std::vector<std::unique_ptr<T>> &tables)
{
    for (auto &p : tables) {
        T &t = *p;
        t.last = &p == &tables.back();
        t.shift = 0;
        while (t.units > 0 && (t.units - 1) >> t.shift >= kHints) ++t.shift;
        int k = 0;
        for (uint32_t j = 0; j < kHints + 2; ++j) {
            while (k + 1 < t.n && t.e[k].end <= (uint64_t)j << t.shift) ++k;
            t.hint[j] = (uint16_t)k;
        }
    }
}

void add_grad(aspis_tensors &list, const void *in, void *out, int64_t numel, int type, int out_type)
{
    GradEntry e = {};
    e.in = in;
    e.out = out;
    e.length_types = (uint64_t)numel | (uint64_t)type << 48 | (uint64_t)out_type << 56;
    append<GradTable, GradEntry, kGrads>(list.tables, e, units_of(numel, grad_unit(type)), list.n);
    ++list.n;
}

void finish(aspis_tensors &list)
{
    if (list.tables.empty()) list.tables.push_back(std::make_unique<GradTable>());      // an empty list's norm is 0
    finish(list.tables);
    for (auto &t : list.tables)
        t->in_place = std::all_of(t->e, t->e + t->n, [](const GradEntry &e) { return e.in == e.out; });
}

aspis_status make_tensors(const aspis_tensor *t, int64_t n, aspis_tensors &list)
{
    Ranges written;
    for (int64_t i = 0; i < n; ++i) {
        aspis_status s = check_array(t[i].data, t[i].numel, t[i].type);
        if (s == ASPIS_OK && t[i].out) s = check_array(t[i].out, t[i].numel, t[i].out_type);
        if (s != ASPIS_OK) return s;
        const bool in_place = !t[i].out || (t[i].out == t[i].data && t[i].out_type == t[i].type);
        const int out_type = in_place ? t[i].type : t[i].out_type;
        written.add(t[i].data, t[i].numel * type_bytes(t[i].type), in_place);
        if (!in_place) written.add(t[i].out, t[i].numel * type_bytes(out_type), true);
        add_grad(list, t[i].data, in_place ? t[i].data : t[i].out, t[i].numel, t[i].type, out_type);
    }
    list.apart = written.apart();
    finish(list);
    return ASPIS_OK;
}

aspis_status make_params(const aspis_param *p, int64_t n, aspis_params &list)
{
    Ranges written;
    for (int64_t i = 0; i < n; ++i) {
        const aspis_param &x = p[i];
        aspis_status s = check_array(x.param, x.numel, x.param_type);
        if (s == ASPIS_OK) s = check_array(x.grad, x.numel, x.grad_type);
        if (s == ASPIS_OK) s = check_array(x.exp_avg, x.numel, ASPIS_F32);
        if (s == ASPIS_OK) s = check_array(x.exp_avg_sq, x.numel, ASPIS_F32);
        if (s == ASPIS_OK && x.master) s = check_array(x.master, x.numel, ASPIS_F32);
        if (s != ASPIS_OK) return s;
        if (x.master && x.param_type == ASPIS_F32) return ASPIS_E_INVAL;
        if (!(x.weight_decay >= 0.0f) || isinf(x.weight_decay) || x.reserved != 0) return ASPIS_E_INVAL;
        written.add(x.param, x.numel * type_bytes(x.param_type), true);
        written.add(x.grad, x.numel * type_bytes(x.grad_type), false);
        written.add(x.exp_avg, x.numel * 4, true);
        written.add(x.exp_avg_sq, x.numel * 4, true);
        if (x.master) written.add(x.master, x.numel * 4, true);
        add_grad(list.grads, x.grad, nullptr, x.numel, x.grad_type, x.grad_type);
    }
    if (!written.apart()) return ASPIS_E_INVAL;
    finish(list.grads);
    list.n = n;
    for (int64_t i = 0; i < n; ++i) {
        const aspis_param &x = p[i];
        if (x.numel == 0) continue;
        auto g = std::find_if(list.groups.begin(), list.groups.end(), [&](const aspis_params::Group &k) {
            return k.param_type == x.param_type && k.grad_type == x.grad_type && k.master == (x.master != nullptr);
        });
        if (g == list.groups.end()) {
            list.groups.push_back({x.param_type, x.grad_type, x.master != nullptr, {}});
            g = list.groups.end() - 1;
        }
        ParamEntry e = {};
        e.param = x.param;
        e.master = x.master;
        e.grad = x.grad;
        e.m = x.exp_avg;
        e.v = x.exp_avg_sq;
        e.numel = x.numel;
        e.decay = x.weight_decay;
        append<ParamTable, ParamEntry, kParams>(g->tables, e, units_of(x.numel, kParamUnit), i);
    }
    for (auto &g : list.groups) finish(g.tables);
    return ASPIS_OK;
}

// n descriptions -> a list in *out; no exception leaves
template <class D, class L>
aspis_status create(const D *d, int64_t n, L **out, aspis_status (*make)(const D *, int64_t, L &))
{
    if (!out) return ASPIS_E_INVAL;
    *out = nullptr;
    if (n < 0 || (n > 0 && !d)) return ASPIS_E_INVAL;
    if (n > (1 << 24)) return ASPIS_E_RANGE;
    try {
        auto list = std::make_unique<L>();
        const aspis_status s = make(d, n, *list);
        if (s == ASPIS_OK) *out = list.release();
        return s;
    } catch (const std::bad_alloc &) {
        return ASPIS_E_RANGE;
    }
}

}  // namespace

extern "C" aspis_status aspis_tensors_create(const aspis_tensor *tensors, int64_t n, aspis_tensors **out)
{
    return create(tensors, n, out, make_tensors);
}

extern "C" void aspis_tensors_destroy(aspis_tensors *list) { delete list; }

extern "C" aspis_status aspis_params_create(const aspis_param *params, int64_t n, aspis_params **out)
{
    return create(params, n, out, make_params);
}

extern "C" void aspis_params_destroy(aspis_params *list) { delete list; }
