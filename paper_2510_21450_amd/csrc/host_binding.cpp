// The host path of the Python entry points that sit in a model's inner loop: argument checks, output and
// workspace allocation, the call into the library and the autograd nodes, in native code.  A short solve takes the
// device about 10 us; checks, allocations and ctypes marshalling in Python took 15 us of host time on top of the call.
// No arithmetic here, and no device code: everything runs in the kernels behind pararnn.h.
#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/StreamGuard.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/accumulate_grad.h>
#include <torch/csrc/utils/pybind.h>
#include <torch/custom_class.h>

#include <algorithm>
#include <array>
#include <map>
#include <mutex>
#include <string>
#include <vector>

#include "pararnn.h"

namespace py = pybind11;
using at::Tensor;
using OptTensor = c10::optional<Tensor>;

namespace {

// Entry points of a cell: the built-in ones with the cell number bound, or those of a library made with
// PARARNN_DEFINE_CELL (addresses).
struct Cell : torch::CustomClassHolder {
    using Ws = size_t (*)(int, int, int, int, int);
    using Fwd = int (*)(int, const float *, const void *, const void *, int, int, int, float, int, void *, int *, float *,
                        void *, size_t, void *);
    using Bwd = int (*)(int, const float *, const void *, const void *, const void *, const void *, int, int, int, void *,
                        float *, void *, void *, size_t, void *);
    using Parts = size_t (*)(int, int, int, int, int, int, size_t *);
    int number = -1, G = 0, S = 0;
    bool keeps_small = false;      // whether a workspace is kept for problems of any size
    std::string what;
    Ws ws_fn = nullptr, ws_fused_fn = nullptr;
    Parts parts_fn = nullptr;      // not in a library built before there was one
    int (*tiles_fn)(int, int, int, int) = nullptr;      // tiles along L, where records depend on L by their number alone
    Fwd fwd_fn = nullptr;
    Bwd bwd_fn = nullptr;

    size_t ws(int dt, int B, int L, int H, int back) const
    {
        return number >= 0 ? pararnn_workspace_bytes(number, dt, B, L, H, back) : ws_fn(dt, B, L, H, back);
    }
    size_t ws_fused(int dt, int B, int L, int H, int n) const
    {
        return number >= 0 ? pararnn_workspace_bytes_fused(number, dt, B, L, H, n) : ws_fused_fn(dt, B, L, H, n);
    }
    size_t parts(int dt, int B, int L, int H, int back, int n, size_t *rest) const
    {
        if (number >= 0) return pararnn_workspace_parts(number, dt, B, L, H, back, n, rest);
        return parts_fn ? parts_fn(dt, B, L, H, back, n, rest) : 0;
    }
};
using CellPtr = c10::intrusive_ptr<Cell>;

const char *type_name(at::ScalarType t)
{
    return t == at::kFloat ? "torch.float32" : t == at::kBFloat16 ? "torch.bfloat16" : t == at::kInt ? "torch.int32" : c10::toString(t);
}

std::string shape_str(at::IntArrayRef s)
{
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + (s.size() == 1 ? ",)" : ")");
}

void check(const Tensor &t, const char *name, at::ScalarType dtype)
{
    if (!t.is_cuda()) throw py::value_error(std::string(name) + " must be a CUDA tensor");
    if (t.scalar_type() != dtype)
        throw py::value_error(std::string(name) + " must be " + type_name(dtype) + ", got " + type_name(t.scalar_type()));
    if (!t.is_contiguous()) throw py::value_error(std::string(name) + " must be contiguous");
}
void check(const Tensor &t, const char *name, at::ScalarType dtype, at::IntArrayRef shape)
{
    check(t, name, dtype);
    if (t.sizes() != shape)
        throw py::value_error(std::string(name) + " must have shape " + shape_str(shape) + ", got " + shape_str(t.sizes()));
}

int dtype_code(at::ScalarType t)
{
    if (t == at::kFloat) return PARARNN_F32;
    if (t == at::kBFloat16) return PARARNN_BF16;
    throw py::key_error(type_name(t));
}

bool has(const OptTensor &t) { return t.has_value() && t->defined(); }
void *ptr(const OptTensor &t) { return has(t) ? t->data_ptr() : nullptr; }
void *stream_ptr(const c10::optional<int64_t> &stream)
{
    return stream ? reinterpret_cast<void *>(*stream) : static_cast<void *>(c10::hip::getCurrentHIPStream().stream());
}
void raise_if(int code, const std::string &what)
{
    if (code != 0)
        throw std::runtime_error(what + " failed: " + pararnn_status_string(code) + " (" + std::to_string(code) + ")");
}
// (a workspace of host memory or of another device would hand the kernels an address that is not theirs)
Tensor workspace_of(size_t bytes, const Tensor &like, const OptTensor &given)
{
    if (has(given) && given->device() != like.device())
        throw py::value_error("workspace must be on " + like.device().str() + ", got " + given->device().str());
    return has(given) ? *given : at::empty({(int64_t)(bytes > 256 ? bytes : 256)}, like.options().dtype(at::kByte));
}

struct Dims { int B, L, H; };

// ------------------------------------------------------------------ kept workspaces
// The carry records of a solve or a backward pass have to be cleared unless the library knows what they hold: 1.3 GB for
// 2^30 timestep-channels (0.25 ms of a forward solve, 0.05 of a backward pass and, in small passes, a launch of 5 us).  So
// the fronts of the workspaces (control block and records) of the diagonal cells' calls are kept between calls, per device,
// stream and problem, under the library's per-workspace promise; what nothing reads after the call (boundary rows, the fp32
// iterate of bf16 storage, sums of parameter gradients: three quarters of a bf16 solve's workspace) is allocated for each
// call as before.  A call takes a front out while it enqueues its work, and the next one that gets it is behind it in the
// same stream; calls of several threads find different ones.  Bounds per device: kMost fronts of the solvers, as many of the gated
// recurrence (whose small ones would else push those out) and a thirty-second of its
// memory, the least recently used go first, and all of them when torch's allocator would take more memory (GiveBack).  Under stream
// capture, with a workspace or a stream of the caller's, for small problems (0.5 us of host time to look would show there; not
// those of the gated recurrence, where clearing is a launch more) and for kernels without records nothing is kept.
using WsKey = std::array<int64_t, 8>;
constexpr size_t kMost = 16;
constexpr double kSmall = 1 << 20;       // timestep-channels; below, most calls take kernels without records and 10-20 us
struct KeptWs { WsKey key; Tensor ws; bool gated; };
struct DevicePool {
    std::vector<KeptWs> free;          // least recently used first
    size_t bytes = 0, cap = 0;
};
std::mutex &pool_mutex()
{
    static std::mutex &m = *new std::mutex;
    return m;
}
std::map<int, DevicePool> &pools()
{
    static std::map<int, DevicePool> &p = *new std::map<int, DevicePool>;     // never destroyed: the runtime may be gone by then
    return p;
}

// Part of a workspace, allocated while its size is known to GiveBack.
thread_local size_t t_allocating = 0;
Tensor own_memory(size_t bytes, const Tensor &like)
{
    struct Note {
        explicit Note(size_t n) { t_allocating = n; }
        ~Note() { t_allocating = 0; }
    } note(bytes);
    return workspace_of(bytes, like, {});
}

// Gives a kept workspace up; the device is the current one.  The library has to know before the memory goes.
void give_up(Tensor &ws)
{
    pararnn_workspace_keep(ws.data_ptr(), 0);
    ws.reset();
}

class Workspace {
public:
    // n_iters: of a fixed-count solve, else 0; bytes: of a whole workspace
    Workspace(const Cell &c, bool back, int code, const Dims &d, int64_t n_iters, size_t bytes, const Tensor &like,
              const OptTensor &given, const c10::optional<int64_t> &stream)
    {
        size_t rest = 0;
        const size_t front = has(given) || stream ? 0 : look(c, back, code, d, n_iters, like, &rest);
        if (device_ < 0) { ws_ = workspace_of(bytes, like, given); return; }
        if (!kept_) {
            ws_ = own_memory(front, like);
            kept_ = pararnn_workspace_keep(ws_.data_ptr(), 1) == PARARNN_OK;
        }
        if (rest == 0) return;
        try {
            rest_ = own_memory(rest, like);
        } catch (...) {
            if (kept_) give_up(ws_);         // no destructor runs for an object that was not constructed
            throw;
        }
        pararnn_workspace_rest(ws_.data_ptr(), rest_.data_ptr(), (size_t)rest_.numel());
    }
    Workspace(const Workspace &) = delete;
    Workspace &operator=(const Workspace &) = delete;
    // after a call that failed, or one without carry records
    ~Workspace() { if (kept_) give_up(ws_); }

    void *data() const { return ws_.data_ptr(); }
    size_t size() const { return (size_t)ws_.numel(); }
    // the call's work is enqueued
    void done()
    {
        if (!kept_ || !pararnn_workspace_known(ws_.data_ptr())) return;
        std::vector<KeptWs> old;
        {
            std::lock_guard<std::mutex> lock(pool_mutex());
            DevicePool &p = pools()[device_];
            p.bytes += (size_t)ws_.numel();
            p.free.push_back({key_, std::move(ws_), gated_});
            kept_ = false;
            const auto alike = [&](const KeptWs &k) { return k.gated == gated_; };
            const auto too_many = [&] { return (size_t)std::count_if(p.free.begin(), p.free.end(), alike) > kMost; };
            while (too_many() || p.bytes > p.cap) {
                const auto k = too_many() ? std::find_if(p.free.begin(), p.free.end(), alike) : p.free.begin();
                p.bytes -= (size_t)k->ws.numel();
                old.push_back(std::move(*k));
                p.free.erase(k);
            }
        }
        for (KeptWs &k : old) give_up(k.ws);
    }

private:
    // Whether this call's front is one to keep (device_), and a kept one if there is one (ws_, kept_).  Returns its size.
    size_t look(const Cell &c, bool back, int code, const Dims &d, int64_t n_iters, const Tensor &like, size_t *rest)
    {
        if (!c.keeps_small && (double)d.B * d.L * d.H < kSmall) return 0;
        const auto cur = c10::hip::getCurrentHIPStream();
        hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
        if (cur.device_index() != like.get_device() || hipStreamIsCapturing(cur.stream(), &cap) != hipSuccess ||
            cap != hipStreamCaptureStatusNone)
            return 0;
        const size_t front = c.parts(code, d.B, d.L, d.H, back, (int)n_iters, rest);
        if (front == 0) return 0;
        key_ = {reinterpret_cast<int64_t>(cur.stream()), c.number >= 0 ? c.number : reinterpret_cast<int64_t>(c.fwd_fn),
                back ? -1 : n_iters, code, d.B, c.tiles_fn ? c.tiles_fn(code, d.B, d.L, d.H) : d.L, d.H, (int64_t)front};
        gated_ = c.keeps_small;
        std::lock_guard<std::mutex> lock(pool_mutex());
        DevicePool &p = pools()[cur.device_index()];
        if (p.cap == 0) {
            size_t avail = 0, total = 0;
            p.cap = hipMemGetInfo(&avail, &total) == hipSuccess ? total / 32 : 1;
        }
        if (front > p.cap) return 0;
        device_ = cur.device_index();
        for (size_t i = p.free.size(); i-- > 0;)
            if (p.free[i].key == key_) {
                ws_ = std::move(p.free[i].ws);
                p.free.erase(p.free.begin() + (long)i);
                p.bytes -= (size_t)ws_.numel();
                kept_ = true;
                break;
            }
        return front;
    }

    Tensor ws_, rest_;
    WsKey key_{};
    int device_ = -1;
    bool kept_ = false, gated_ = false;
};

// Gives up what is kept on the current device; returns its bytes.
int64_t release_on_device(int device)
{
    std::vector<KeptWs> old;
    int64_t bytes = 0;
    {
        std::lock_guard<std::mutex> lock(pool_mutex());
        const auto p = pools().find(device);
        if (p == pools().end()) return 0;
        bytes = (int64_t)p->second.bytes;
        p->second.bytes = 0;
        old.swap(p->second.free);
    }
    for (KeptWs &k : old) give_up(k.ws);
    return bytes;
}

int64_t release_workspaces()
{
    std::vector<int> devices;
    {
        std::lock_guard<std::mutex> lock(pool_mutex());
        for (auto &p : pools()) devices.push_back(p.first);
    }
    int64_t bytes = 0;
    for (int d : devices) {
        const c10::DeviceGuard guard(c10::Device(c10::DeviceType::CUDA, (c10::DeviceIndex)d));
        bytes += release_on_device(d);
    }
    return bytes;
}

// torch's allocator asks before it takes more memory from the device, and so before an allocation fails; it does not say
// how much it needs.  It gets everything kept on the device it allocates on: the current one, and no other, whose allocator
// may be locked by a thread that waits for this one.  Only a workspace of this thread's own call does not push out the kept
// ones while there is memory for both: forward and backward pass of one training step would otherwise take turns with the
// same memory for good.  The allocator's lock is held here and taken again by what is freed, which it allows; the pool's own
// lock is never held while memory is allocated or freed.
struct GiveBack : c10::FreeMemoryCallback {
    bool Execute() override
    {
        int device = -1;
        hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
        if (hipStreamIsCapturing(c10::hip::getCurrentHIPStream().stream(), &cap) != hipSuccess || cap != hipStreamCaptureStatusNone)
            return false;
        if (hipGetDevice(&device) != hipSuccess) return false;
        size_t avail = 0, total = 0;
        if (t_allocating > 0 && hipMemGetInfo(&avail, &total) == hipSuccess) {
            namespace alloc = c10::hip::HIPCachingAllocator;
            const double need = (double)t_allocating + (32 << 20);        // the allocator rounds up
            const double mine = (double)alloc::getDeviceStats(device).reserved_bytes[0].current;
            if (need <= (double)avail && mine + need <= (double)total * alloc::getMemoryFraction(device)) return false;
        }
        return release_on_device(device) > 0;
    }
};

Dims dims4(const Tensor &u, const char *name)
{
    if (u.dim() != 4) throw py::value_error(std::string(name) + " must have four dimensions");
    return {(int)u.size(0), (int)u.size(1), (int)u.size(3)};
}

struct Solve { Tensor h, iters, trace; };

Solve solve(const Cell &c, const Tensor &params, const Tensor &u, const OptTensor &h0, double tol, int64_t max_iter, bool trace,
            const OptTensor &workspace, const c10::optional<int64_t> &stream, const OptTensor &out)
{
    const Dims d = dims4(u, "u");
    const auto dt = u.scalar_type();
    const int code = dtype_code(dt);
    check(u, "u", dt, {d.B, d.L, c.G, d.H});
    check(params, "params", at::kFloat);
    if (has(h0)) check(*h0, "h0", dt, {d.B, c.S, d.H});
    Solve r;
    r.h = has(out) ? *out : at::empty({d.B, d.L, c.S, d.H}, u.options());
    check(r.h, "h", dt, {d.B, d.L, c.S, d.H});
    r.iters = at::empty({2}, u.options().dtype(at::kInt));
    if (trace) r.trace = at::zeros({max_iter > 1 ? max_iter : 1}, u.options().dtype(at::kFloat));
    const size_t need = tol < 0 ? c.ws_fused(code, d.B, d.L, d.H, (int)max_iter) : c.ws(code, d.B, d.L, d.H, 0);
    Workspace ws(c, false, code, d, tol < 0 ? max_iter : 0, need, u, workspace, stream);
    float *tr = trace ? static_cast<float *>(r.trace.data_ptr()) : nullptr;
    const float *p = static_cast<const float *>(params.data_ptr());
    int *it = static_cast<int *>(r.iters.data_ptr());
    const int rc = c.number >= 0
                       ? pararnn_forward(c.number, code, p, u.data_ptr(), ptr(h0), d.B, d.L, d.H, (float)tol, (int)max_iter,
                                         r.h.data_ptr(), it, tr, ws.data(), ws.size(), stream_ptr(stream))
                       : c.fwd_fn(code, p, u.data_ptr(), ptr(h0), d.B, d.L, d.H, (float)tol, (int)max_iter, r.h.data_ptr(), it,
                                  tr, ws.data(), ws.size(), stream_ptr(stream));
    raise_if(rc, c.what + "_forward");
    ws.done();
    return r;
}

struct Grads { Tensor du, dparams, dh0; };

Grads adjoint(const Cell &c, const Tensor &params, const Tensor &u, const OptTensor &h0, const Tensor &h, const Tensor &g,
              bool want_dh0, const OptTensor &workspace, const c10::optional<int64_t> &stream, const Grads *out)
{
    const Dims d = dims4(u, "u");
    const auto dt = u.scalar_type();
    const int code = dtype_code(dt);
    check(u, "u", dt, {d.B, d.L, c.G, d.H});
    check(params, "params", at::kFloat);
    check(h, "h", dt, {d.B, d.L, c.S, d.H});
    check(g, "dL_dh", dt, {d.B, d.L, c.S, d.H});
    if (has(h0)) check(*h0, "h0", dt, {d.B, c.S, d.H});
    Grads r;
    if (out) {
        r = *out;
        check(r.du, "dL_du", dt, u.sizes());
        check(r.dparams, "dL_dparams", at::kFloat, params.sizes());
        if (r.dh0.defined()) check(r.dh0, "dL_dh0", dt, {d.B, c.S, d.H});
    } else {
        r.du = at::empty(u.sizes(), u.options());
        r.dparams = at::empty(params.sizes(), params.options());
        if (want_dh0) r.dh0 = at::empty({d.B, c.S, d.H}, u.options());
    }
    Workspace ws(c, true, code, d, 0, c.ws(code, d.B, d.L, d.H, 1), u, workspace, stream);
    const float *p = static_cast<const float *>(params.data_ptr());
    float *dp = static_cast<float *>(r.dparams.data_ptr());
    void *dh = r.dh0.defined() ? r.dh0.data_ptr() : nullptr;
    const int rc = c.number >= 0
                       ? pararnn_backward(c.number, code, p, u.data_ptr(), ptr(h0), h.data_ptr(), g.data_ptr(), d.B, d.L, d.H,
                                          r.du.data_ptr(), dp, dh, ws.data(), ws.size(), stream_ptr(stream))
                       : c.bwd_fn(code, p, u.data_ptr(), ptr(h0), h.data_ptr(), g.data_ptr(), d.B, d.L, d.H, r.du.data_ptr(),
                                  dp, dh, ws.data(), ws.size(), stream_ptr(stream));
    raise_if(rc, c.what + "_backward");
    ws.done();
    return r;
}

struct ProjDims { int B, L, H, G; };
ProjDims proj_dims(const Tensor &x, const Tensor &Wx, int64_t n_heads)
{
    if (x.dim() != 3) throw py::value_error("x must have three dimensions");
    if (Wx.dim() < 1) throw py::value_error("Wx must have three dimensions");
    const ProjDims d = {(int)x.size(0), (int)x.size(1), (int)x.size(2), (int)Wx.size(0)};
    check(x, "x", x.scalar_type(), {d.B, d.L, d.H});
    if (n_heads == 0) throw py::value_error("n_heads must be positive");
    check(Wx, "Wx", at::kFloat, {d.G, d.H, d.H / n_heads});
    return d;
}

Tensor project(const Tensor &x, const Tensor &Wx, const OptTensor &bias, int64_t n_heads, const OptTensor &workspace,
               const c10::optional<int64_t> &stream, const OptTensor &out)
{
    const ProjDims d = proj_dims(x, Wx, n_heads);
    const auto dt = x.scalar_type();
    const int code = dtype_code(dt);
    if (has(bias)) check(*bias, "bias", at::kFloat, {d.G, d.H});
    Tensor u = has(out) ? *out : at::empty({d.B, d.L, d.G, d.H}, x.options());
    check(u, "u", dt, {d.B, d.L, d.G, d.H});
    const Tensor ws = workspace_of(pararnn_input_projection_workspace_bytes(code, d.B, d.L, d.H, d.G, (int)n_heads, 0), x, workspace);
    raise_if(pararnn_input_projection(code, x.data_ptr(), static_cast<const float *>(Wx.data_ptr()),
                                      static_cast<const float *>(ptr(bias)), d.B, d.L, d.H, d.G, (int)n_heads, u.data_ptr(),
                                      ws.data_ptr(), (size_t)ws.numel(), stream_ptr(stream)),
             "pararnn_input_projection");
    return u;
}

struct ProjGrads { Tensor dx, dW, db; };

ProjGrads project_backward(const Tensor &x, const Tensor &Wx, const Tensor &du, int64_t n_heads, bool want_dx, bool want_dw,
                           bool want_db, const OptTensor &workspace, const c10::optional<int64_t> &stream)
{
    const ProjDims d = proj_dims(x, Wx, n_heads);
    const auto dt = x.scalar_type();
    const int code = dtype_code(dt);
    check(du, "du", dt, {d.B, d.L, d.G, d.H});
    ProjGrads r;
    if (want_dx) r.dx = at::empty(x.sizes(), x.options());
    if (want_dw) r.dW = at::empty(Wx.sizes(), Wx.options());
    if (want_db) r.db = at::empty({d.G, d.H}, Wx.options());
    const Tensor ws = workspace_of(pararnn_input_projection_workspace_bytes(code, d.B, d.L, d.H, d.G, (int)n_heads, 1), x, workspace);
    auto p = [](const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; };
    raise_if(pararnn_input_projection_backward(code, x.data_ptr(), static_cast<const float *>(Wx.data_ptr()), du.data_ptr(), d.B,
                                               d.L, d.H, d.G, (int)n_heads, p(r.dx), static_cast<float *>(p(r.dW)),
                                               static_cast<float *>(p(r.db)), ws.data_ptr(), (size_t)ws.numel(),
                                               stream_ptr(stream)),
             "pararnn_input_projection_backward");
    return r;
}

// ------------------------------------------------------------------ gated linear recurrence, 4-bit weights
// These calls run on the device of their tensors, whichever is current, and on the caller's stream if there is one: what they
// allocate belongs to the stream that uses it.
class On {
public:
    On(const Tensor &t, const char *name, const c10::optional<int64_t> &stream)
    {
        if (!t.is_cuda()) throw py::value_error(std::string(name) + " must be a CUDA tensor");
        guard_.reset_device(t.device());
        auto s = stream ? c10::hip::getStreamFromExternal(reinterpret_cast<hipStream_t>(*stream), t.get_device())
                        : c10::hip::getCurrentHIPStream(t.get_device());
        if (stream) on_.emplace(s.unwrap());
        stream_ = static_cast<void *>(s.stream());
    }
    void *stream() const { return stream_; }

private:
    c10::OptionalDeviceGuard guard_;
    c10::optional<c10::StreamGuard> on_;
    void *stream_;
};

void check_on(const Tensor &t, const char *name, at::ScalarType dtype, at::IntArrayRef shape, const Tensor &like)
{
    check(t, name, dtype, shape);
    if (t.device() != like.device()) throw py::value_error(std::string(name) + " must be on " + like.device().str() + ", got " + t.device().str());
}

int int_of(int64_t n, const char *name)
{
    if (n < 0 || n > 0x7fffffff) throw py::value_error(std::string(name) + " is out of range");
    return (int)n;
}

struct GatedDims { int B, L, G, H; };
GatedDims gated_dims(const Tensor &u)
{
    if (u.dim() != 4) throw py::value_error("u must have four dimensions");
    const GatedDims d = {int_of(u.size(0), "u"), int_of(u.size(1), "u"), int_of(u.size(2), "u"), int_of(u.size(3), "u")};
    check(u, "u", u.scalar_type());
    if (d.G != 2 && d.G != 3) throw py::value_error("u must have 2 or 3 gates, got " + std::to_string(d.G));
    return d;
}

// The gated calls' kept workspaces: all of it is a front, and the layout is the same for both directions, types and gates.
const Cell &gated_cell()
{
    static Cell &c = *[] {
        static char name;
        Cell *r = new Cell;
        r->what = "pararnn_gated";
        r->fwd_fn = reinterpret_cast<Cell::Fwd>(&name);      // never called: a name no other cell has
        r->keeps_small = true;                               // whatever has records here has several tiles, and clearing is a launch of its own
        r->parts_fn = [](int dtype, int B, int L, int H, int, int, size_t *rest) {
            *rest = 0;
            return pararnn_gated_workspace_bytes(dtype, B, L, H, 2);
        };
        r->tiles_fn = [](int dtype, int B, int L, int H) {   // a checkpoint for each, B x H fp32 numbers
            return (int)(pararnn_gated_checkpoint_bytes(dtype, B, L, H, 2) / 4 / B / H);
        };
        return r;
    }();
    return c;
}
// None (an undefined tensor) where the call uses none.
struct GatedWorkspace {
    GatedWorkspace(const GatedDims &d, int code, const Tensor &like, const OptTensor &given, const c10::optional<int64_t> &stream)
    {
        const size_t bytes = pararnn_gated_workspace_bytes(code, d.B, d.L, d.H, d.G);
        if (has(given)) check_on(*given, "workspace", at::kByte, {given->numel()}, like);
        if (bytes > 256 || has(given)) ws.emplace(gated_cell(), false, PARARNN_F32, Dims{d.B, d.L, d.H}, 0, bytes, like, given, stream);
    }
    void *data() const { return ws ? ws->data() : nullptr; }
    size_t size() const { return ws ? ws->size() : 0; }
    void done() { if (ws) ws->done(); }
    c10::optional<Workspace> ws;
};

struct GatedOut { Tensor h, last, ckpt; };

GatedOut gated_solve(const Tensor &u, const OptTensor &h0, const OptTensor &lengths, bool checkpoints, const OptTensor &workspace,
                     const c10::optional<int64_t> &stream, const OptTensor &out, const OptTensor &out_last)
{
    const On on(u, "u", stream);
    const GatedDims d = gated_dims(u);
    const auto dt = u.scalar_type();
    const int code = dtype_code(dt);
    if (has(h0)) check_on(*h0, "h0", at::kFloat, {d.B, d.H}, u);
    if (has(lengths)) check_on(*lengths, "lengths", at::kInt, {d.B}, u);
    GatedOut r;
    r.h = has(out) ? *out : at::empty({d.B, d.L, d.H}, u.options());
    check_on(r.h, "h", dt, {d.B, d.L, d.H}, u);
    r.last = has(out_last) ? *out_last : at::empty({d.B, d.H}, u.options().dtype(at::kFloat));
    check_on(r.last, "h_last", at::kFloat, {d.B, d.H}, u);
    if (checkpoints) {
        const size_t bytes = pararnn_gated_checkpoint_bytes(code, d.B, d.L, d.H, d.G);
        const int64_t rows = bytes ? (int64_t)(bytes / 4 / d.B / d.H) : 0;
        r.ckpt = at::empty({d.B, rows, d.H}, u.options().dtype(at::kFloat));
    }
    GatedWorkspace ws(d, code, u, workspace, stream);
    raise_if(pararnn_gated_forward(code, u.data_ptr(), static_cast<const float *>(ptr(h0)), static_cast<const int *>(ptr(lengths)), d.B,
                                   d.L, d.H, d.G, r.h.data_ptr(), static_cast<float *>(r.last.data_ptr()),
                                   checkpoints ? static_cast<float *>(r.ckpt.data_ptr()) : nullptr, ws.data(), ws.size(), on.stream()),
             "pararnn_gated_forward");
    ws.done();
    return r;
}

struct GatedGrads { Tensor du, dh0; };

GatedGrads gated_adjoint(const Tensor &u, const Tensor &ckpt, const OptTensor &g, const OptTensor &dlast, const OptTensor &lengths,
                         bool want_dh0, const OptTensor &workspace, const c10::optional<int64_t> &stream, const OptTensor &out)
{
    const On on(u, "u", stream);
    const GatedDims d = gated_dims(u);
    const auto dt = u.scalar_type();
    const int code = dtype_code(dt);
    const size_t bytes = pararnn_gated_checkpoint_bytes(code, d.B, d.L, d.H, d.G);
    check_on(ckpt, "checkpoints", at::kFloat, {d.B, bytes ? (int64_t)(bytes / 4 / d.B / d.H) : 0, d.H}, u);
    if (has(g)) check_on(*g, "dL_dh", dt, {d.B, d.L, d.H}, u);
    if (has(dlast)) check_on(*dlast, "dL_dlast", at::kFloat, {d.B, d.H}, u);
    if (has(lengths)) check_on(*lengths, "lengths", at::kInt, {d.B}, u);
    GatedGrads r;
    r.du = has(out) ? *out : at::empty(u.sizes(), u.options());
    check_on(r.du, "dL_du", dt, u.sizes(), u);
    if (want_dh0) r.dh0 = at::empty({d.B, d.H}, u.options().dtype(at::kFloat));
    GatedWorkspace ws(d, code, u, workspace, stream);
    raise_if(pararnn_gated_backward(code, u.data_ptr(), static_cast<const float *>(ckpt.data_ptr()), static_cast<const int *>(ptr(lengths)),
                                    ptr(g), static_cast<const float *>(ptr(dlast)), d.B, d.L, d.H, d.G, r.du.data_ptr(),
                                    want_dh0 ? static_cast<float *>(r.dh0.data_ptr()) : nullptr, ws.data(), ws.size(), on.stream()),
             "pararnn_gated_backward");
    ws.done();
    return r;
}

// 4-bit weights as the Python side holds them
struct Q4 {
    Tensor packed, scales;
    int G, H, heads, group;
};

struct Q4Shape { int G, H, dh, heads; };
Q4Shape q4_shape(const Tensor &W, const char *name, at::ScalarType dtype, int64_t n_heads)
{
    if (W.dim() != 3) throw py::value_error(std::string(name) + " must have three dimensions");
    if (n_heads < 1) throw py::value_error("n_heads must be positive");
    const Q4Shape s = {int_of(W.size(0), name), int_of(W.size(1), name), int_of(W.size(1) / n_heads, name), int_of(n_heads, "n_heads")};
    check(W, name, dtype, {s.G, s.H, s.dh});
    if ((int64_t)s.dh * n_heads != s.H) throw py::value_error("n_heads must divide H");
    return s;
}

Q4 q4_empty(const Q4Shape &s, int64_t group, const Tensor &like)
{
    Q4 q;
    q.G = s.G; q.H = s.H; q.heads = s.heads; q.group = int_of(group, "group");
    q.packed = at::empty({(int64_t)pararnn_q4_packed_bytes(s.H, s.G, s.heads)}, like.options().dtype(at::kByte));
    q.scales = at::empty({(int64_t)pararnn_q4_scale_bytes(s.H, s.G, s.heads, q.group) / 2}, like.options().dtype(at::kBFloat16));
    return q;
}

// Refuses what the library would before anything is allocated: an empty buffer has no address.
void q4_supported(const Q4Shape &s, int64_t group)
{
    if (group != 32 && group != 64 && group != 128) throw py::value_error("group must be 32, 64 or 128, got " + std::to_string(group));
    if (s.G < 1 || s.G > 8) throw py::value_error("there must be 1 to 8 gates, got " + std::to_string(s.G));
    if (pararnn_q4_scale_bytes(s.H, s.G, s.heads, (int)group) == 0)
        throw py::value_error("channels per head must be a multiple of 64 and of group, H at most 1048576");
}

Q4 q4_quantize(const Tensor &W, int64_t n_heads, int64_t group, const c10::optional<int64_t> &stream)
{
    const On on(W, "Wx", stream);
    const Q4Shape s = q4_shape(W, "Wx", at::kFloat, n_heads);
    q4_supported(s, group);
    Q4 q = q4_empty(s, group, W);
    raise_if(pararnn_q4_quantize(static_cast<const float *>(W.data_ptr()), s.H, s.G, s.heads, q.group, q.packed.data_ptr(),
                                 q.scales.data_ptr(), on.stream()),
             "pararnn_q4_quantize");
    return q;
}

Q4 q4_pack(const Tensor &codes, const Tensor &scales, int64_t n_heads, const c10::optional<int64_t> &stream)
{
    const On on(codes, "codes", stream);
    const Q4Shape s = q4_shape(codes, "codes", at::kChar, n_heads);
    const int64_t n = scales.dim() == 3 ? scales.size(2) : 0, group = n > 0 && s.dh % n == 0 ? s.dh / n : 0;
    q4_supported(s, group);
    check_on(scales, "scales", at::kBFloat16, {s.G, s.H, n}, codes);
    Q4 q = q4_empty(s, group, codes);
    raise_if(pararnn_q4_pack(static_cast<const signed char *>(codes.data_ptr()), scales.data_ptr(), s.H, s.G, s.heads, q.group,
                             q.packed.data_ptr(), q.scales.data_ptr(), on.stream()),
             "pararnn_q4_pack");
    return q;
}

void q4_check(const Q4 &q, const Tensor &like)
{
    check_on(q.packed, "packed", at::kByte, {(int64_t)pararnn_q4_packed_bytes(q.H, q.G, q.heads)}, like);
    check_on(q.scales, "scales", at::kBFloat16, {(int64_t)pararnn_q4_scale_bytes(q.H, q.G, q.heads, q.group) / 2}, like);
}

Tensor q4_dequantize(const Q4 &q, const c10::optional<int64_t> &stream)
{
    const On on(q.packed, "packed", stream);
    q4_check(q, q.packed);
    Tensor W = at::empty({q.G, q.H, q.H / q.heads}, q.packed.options().dtype(at::kFloat));
    raise_if(pararnn_q4_dequantize(q.packed.data_ptr(), q.scales.data_ptr(), q.H, q.G, q.heads, q.group,
                                   static_cast<float *>(W.data_ptr()), on.stream()),
             "pararnn_q4_dequantize");
    return W;
}

Tensor q4_project(const Tensor &x, const Q4 &q, const OptTensor &bias, const OptTensor &workspace, const c10::optional<int64_t> &stream,
                  const OptTensor &out)
{
    const On on(x, "x", stream);
    if (x.dim() != 3) throw py::value_error("x must have three dimensions");
    const auto dt = x.scalar_type();
    const int code = dtype_code(dt), B = int_of(x.size(0), "x"), L = int_of(x.size(1), "x");
    check(x, "x", dt, {B, L, q.H});
    q4_check(q, x);
    if (has(bias)) check_on(*bias, "bias", at::kFloat, {q.G, q.H}, x);
    Tensor u = has(out) ? *out : at::empty({B, L, q.G, q.H}, x.options());
    check_on(u, "u", dt, {B, L, q.G, q.H}, x);
    if (has(workspace)) check_on(*workspace, "workspace", at::kByte, {workspace->numel()}, x);
    // (two bytes a weight, which only rounded weights use)
    Tensor ws = has(workspace) ? *workspace : Tensor();
    if (!ws.defined() && pararnn_q4_products() == 1)
        ws = workspace_of(pararnn_q4_workspace_bytes(code, B, L, q.H, q.G, q.heads, q.group), x, {});
    raise_if(pararnn_input_projection_q4(code, x.data_ptr(), q.packed.data_ptr(), q.scales.data_ptr(), static_cast<const float *>(ptr(bias)),
                                         B, L, q.H, q.G, q.heads, q.group, u.data_ptr(), ws.defined() ? ws.data_ptr() : nullptr,
                                         ws.defined() ? (size_t)ws.numel() : 0, on.stream()),
             "pararnn_input_projection_q4");
    return u;
}

struct StepOut { Tensor y, h; };

StepOut gated_step(const Tensor &x, const Q4 &q, const OptTensor &h, const OptTensor &bias, const c10::optional<int64_t> &stream,
                   const OptTensor &out, const OptTensor &out_h)
{
    const On on(x, "x", stream);
    if (x.dim() != 2) throw py::value_error("x must have two dimensions");
    const auto dt = x.scalar_type();
    const int code = dtype_code(dt), B = int_of(x.size(0), "x");
    check(x, "x", dt, {B, q.H});
    q4_check(q, x);
    if (q.G != 2 && q.G != 3) throw py::value_error("the weights must have 2 or 3 gates, got " + std::to_string(q.G));
    if (has(h)) check_on(*h, "h", at::kFloat, {B, q.H}, x);
    if (has(bias)) check_on(*bias, "bias", at::kFloat, {q.G, q.H}, x);
    StepOut r;
    r.y = has(out) ? *out : at::empty({B, q.H}, x.options());
    check_on(r.y, "y", dt, {B, q.H}, x);
    r.h = has(out_h) ? *out_h : at::empty({B, q.H}, x.options().dtype(at::kFloat));
    check_on(r.h, "h_next", at::kFloat, {B, q.H}, x);
    raise_if(pararnn_gated_layer_step(code, x.data_ptr(), q.packed.data_ptr(), q.scales.data_ptr(), static_cast<const float *>(ptr(bias)),
                                      static_cast<const float *>(ptr(h)), B, q.H, q.G, q.heads, q.group, r.y.data_ptr(),
                                      static_cast<float *>(r.h.data_ptr()), on.stream()),
             "pararnn_gated_layer_step");
    return r;
}

// ------------------------------------------------------------------ autograd
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

// Numbers the defined tensors among a function's inputs as the graph does.
struct Edges {
    AutogradContext *ctx;
    size_t next = 0;
    bool operator()(bool defined) { return defined && ctx->needs_input_grad(next++); }
};

Tensor or_none(const OptTensor &t) { return has(t) ? *t : Tensor(); }

// h = RNN(u): pararnn_forward with pararnn_backward as its gradient (Eq. (6)).
struct Recurrence : torch::autograd::Function<Recurrence> {
    static variable_list forward(AutogradContext *ctx, Tensor params, Tensor u, OptTensor h0, CellPtr cell, double tol, int64_t max_iter)
    {
        Solve s = solve(*cell, params, u, h0, tol, max_iter, false, {}, {}, {});
        ctx->save_for_backward({params, u, or_none(h0), s.h});
        ctx->saved_data["cell"] = c10::IValue::make_capsule(cell);
        ctx->mark_non_differentiable({s.iters});
        ctx->set_materialize_grads(false);
        return {s.h, s.iters};
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        variable_list out(6);
        if (!grads[0].defined()) return out;
        const auto v = ctx->get_saved_variables();
        const auto cell = c10::static_intrusive_pointer_cast<Cell>(ctx->saved_data["cell"].toCapsule());
        Edges need{ctx};
        need(true); need(true);
        Grads g = adjoint(*cell, v[0], v[1], v[2], v[3], grads[0].contiguous(), need(v[2].defined()), {}, {}, nullptr);
        out[0] = g.dparams; out[1] = g.du; out[2] = g.dh0;
        return out;
    }
};

// u = B x + b for all gates
struct Projection : torch::autograd::Function<Projection> {
    static variable_list forward(AutogradContext *ctx, Tensor x, Tensor Wx, OptTensor bias, int64_t n_heads)
    {
        Tensor u = project(x, Wx, bias, n_heads, {}, {}, {});
        ctx->save_for_backward({x, Wx});
        ctx->saved_data["n_heads"] = n_heads;
        ctx->saved_data["bias"] = has(bias);
        ctx->set_materialize_grads(false);
        return {u};
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        variable_list out(4);
        if (!grads[0].defined()) return out;
        const auto v = ctx->get_saved_variables();
        Edges need{ctx};
        const bool nx = need(true), nw = need(true), nb = need(ctx->saved_data["bias"].toBool());
        ProjGrads g = project_backward(v[0], v[1], grads[0].contiguous(), ctx->saved_data["n_heads"].toInt(), nx, nw || nb, nb, {}, {});
        out[0] = g.dx;
        if (nw) out[1] = g.dW;
        out[2] = g.db;
        return out;
    }
};

// The projection followed by the recurrence, as one node.
struct Layer : torch::autograd::Function<Layer> {
    static variable_list forward(AutogradContext *ctx, Tensor x, Tensor Wx, OptTensor bias, Tensor params, OptTensor h0, CellPtr cell,
                                 int64_t n_heads, double tol, int64_t max_iter)
    {
        Tensor u = project(x, Wx, bias, n_heads, {}, {}, {});
        Solve s = solve(*cell, params, u, h0, tol, max_iter, false, {}, {}, {});
        ctx->save_for_backward({x, Wx, params, or_none(h0), u, s.h});
        ctx->saved_data["cell"] = c10::IValue::make_capsule(cell);
        ctx->saved_data["n_heads"] = n_heads;
        ctx->saved_data["bias"] = has(bias);
        ctx->mark_non_differentiable({s.iters});
        ctx->set_materialize_grads(false);
        return {s.h, s.iters};
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        variable_list out(9);
        if (!grads[0].defined()) return out;
        const auto v = ctx->get_saved_variables();
        const auto cell = c10::static_intrusive_pointer_cast<Cell>(ctx->saved_data["cell"].toCapsule());
        Edges need{ctx};
        const bool nx = need(true), nw = need(true), nb = need(ctx->saved_data["bias"].toBool());
        need(true);
        Grads g = adjoint(*cell, v[2], v[4], v[3], v[5], grads[0].contiguous(), need(v[3].defined()), {}, {}, nullptr);
        out[3] = g.dparams;
        out[4] = g.dh0;
        if (nx || nw || nb) {
            ProjGrads p = project_backward(v[0], v[1], g.du, ctx->saved_data["n_heads"].toInt(), nx, nw || nb, nb, {}, {});
            out[0] = p.dx;
            if (nw) out[1] = p.dW;
            out[2] = p.db;
        }
        return out;
    }
};

// A backward pass that is captured into a graph while another graph, built on another stream, keeps the accumulators of the same
// leaves alive: the engine would make that stream wait for the captured one, which draws it into the capture and ends the
// process when the capture ends.  Refused before anything is launched; what this node returns is what it would wait for.
// They are found by the node's own edges: its inputs need not be kept for it.
void refuse_foreign_leaves()
{
    const auto cur = c10::hip::getCurrentHIPStream();
    hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
    if (hipStreamIsCapturing(cur.stream(), &cap) != hipSuccess || cap == hipStreamCaptureStatusNone) return;
    for (const torch::autograd::Edge &e : torch::autograd::get_current_node()->next_edges()) {
        if (!dynamic_cast<torch::autograd::AccumulateGrad *>(e.function.get())) continue;
        const auto stream = e.function->stream();
        // (by number: the same stream is of another device type by name in either half of torch)
        if (stream && (stream->id() != cur.id() || stream->device_index() != cur.device_index()))
            throw std::runtime_error("a backward pass cannot be captured into a graph while an eager graph of the same leaves is alive: "
                                     "release that graph (its outputs) first");
    }
}

// Gradients of a backward pass that itself is recorded (create_graph): the kernels' results have no history, so a node that says so
// is put between them and what they depend on, the inputs of the node they are of and its gradients, and a derivative of them is an
// error in place of a missing term.
struct NoSecond : torch::autograd::Node {
    using Node::Node;
    variable_list apply(variable_list &&) override { throw std::runtime_error("the gated recurrence has no second derivatives"); }
};
void once(variable_list &out, const variable_list &grads)
{
    if (!at::GradMode::is_enabled()) return;
    torch::autograd::edge_list on = torch::autograd::get_current_node()->next_edges();
    for (const Tensor &t : grads)
        if (t.defined() && t.requires_grad()) on.push_back(torch::autograd::impl::gradient_edge(t));
    const auto node = std::make_shared<NoSecond>(std::move(on));
    for (Tensor &t : out)
        if (t.defined()) torch::autograd::create_gradient_edge(t, node);
}

// The gated linear recurrence: gated_forward with gated_backward as its gradient.
struct Gated : torch::autograd::Function<Gated> {
    static variable_list forward(AutogradContext *ctx, Tensor u, OptTensor h0, OptTensor lengths, bool train)
    {
        GatedOut r = gated_solve(u, h0, lengths, train, {}, {}, {}, {});
        if (train) ctx->save_for_backward({u, r.ckpt, or_none(lengths)});      // the states in front are in the checkpoints
        ctx->saved_data["h0"] = has(h0);
        ctx->set_materialize_grads(false);
        return {r.h, r.last};
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        variable_list out(4);
        if (!grads[0].defined() && !grads[1].defined()) return out;
        const auto v = ctx->get_saved_variables();
        refuse_foreign_leaves();
        Edges need{ctx};
        need(true);
        const bool nh = need(ctx->saved_data["h0"].toBool());
        GatedGrads g = gated_adjoint(v[0], v[1], dense(grads[0]), dense(grads[1]), v[2], nh, {}, {}, {});
        out[0] = g.du; out[1] = g.dh0;
        once(out, grads);
        return out;
    }
    static OptTensor dense(const Tensor &g) { return g.defined() ? OptTensor(g.contiguous()) : OptTensor(); }
};

// The projection followed by the gated linear recurrence, as one node.
struct GatedLayer : torch::autograd::Function<GatedLayer> {
    static variable_list forward(AutogradContext *ctx, Tensor x, Tensor Wx, OptTensor bias, OptTensor h0, OptTensor lengths, int64_t n_heads,
                                 bool train)
    {
        const On on(x, "x", {});
        for (const OptTensor &t : {OptTensor(Wx), bias})
            if (has(t) && t->device() != x.device()) throw py::value_error("x, Wx and bias must be on one device");
        Tensor u = project(x, Wx, bias, n_heads, {}, {}, {});
        GatedOut r = gated_solve(u, h0, lengths, train, {}, {}, {}, {});
        if (train) ctx->save_for_backward({x, Wx, u, r.ckpt, or_none(lengths)});
        ctx->saved_data["n_heads"] = n_heads;
        ctx->saved_data["bias"] = has(bias);
        ctx->saved_data["h0"] = has(h0);
        ctx->set_materialize_grads(false);
        return {r.h, r.last};
    }
    static variable_list backward(AutogradContext *ctx, variable_list grads)
    {
        variable_list out(7);
        if (!grads[0].defined() && !grads[1].defined()) return out;
        const auto v = ctx->get_saved_variables();
        const On on(v[0], "x", {});
        refuse_foreign_leaves();
        Edges need{ctx};
        const bool nx = need(true), nw = need(true), nb = need(ctx->saved_data["bias"].toBool()), nh = need(ctx->saved_data["h0"].toBool());
        GatedGrads g = gated_adjoint(v[2], v[3], Gated::dense(grads[0]), Gated::dense(grads[1]), v[4], nh, {}, {}, {});
        out[3] = g.dh0;
        if (nx || nw || nb) {
            ProjGrads p = project_backward(v[0], v[1], g.du, ctx->saved_data["n_heads"].toInt(), nx, nw || nb, nb, {}, {});
            out[0] = p.dx;
            if (nw) out[1] = p.dW;
            out[2] = p.db;
        }
        once(out, grads);
        return out;
    }
};

bool wants_grad(std::initializer_list<const OptTensor *> ts)
{
    if (!at::GradMode::is_enabled()) return false;
    for (const OptTensor *t : ts)
        if (has(*t) && (*t)->requires_grad()) return true;
    return false;
}

// Runs a call into the library without the interpreter lock: it may allocate, and wait for a place in a full launch queue.
template <class F> auto unlocked(F &&f)
{
    const py::gil_scoped_release unlock;
    return f();
}

py::object object_of(const Tensor &t) { return t.defined() ? py::cast(t) : py::none(); }

}  // namespace

namespace c10 {
C10_REGISTER_CLASS(FreeHipMemoryCallbacksRegistry, pararnn_kept_workspaces, GiveBack)
}

PYBIND11_MODULE(_host, m)
{
    py::class_<Cell, CellPtr>(m, "Cell");
    m.def("builtin_cell", [](int number, std::string what) {
        auto c = c10::make_intrusive<Cell>();
        c->number = number;
        c->G = pararnn_cell_gates(number);
        c->S = pararnn_cell_state(number);
        c->what = std::move(what);
        return c;
    });
    m.def("library_cell", [](std::string what, int G, int S, size_t ws, size_t ws_fused, size_t fwd, size_t bwd, size_t parts) {
        auto c = c10::make_intrusive<Cell>();
        c->G = G;
        c->S = S;
        c->what = std::move(what);
        c->ws_fn = reinterpret_cast<Cell::Ws>(ws);
        c->ws_fused_fn = reinterpret_cast<Cell::Ws>(ws_fused);
        c->fwd_fn = reinterpret_cast<Cell::Fwd>(fwd);
        c->bwd_fn = reinterpret_cast<Cell::Bwd>(bwd);
        c->parts_fn = reinterpret_cast<Cell::Parts>(parts);
        return c;
    }, py::arg("what"), py::arg("G"), py::arg("S"), py::arg("ws"), py::arg("ws_fused"), py::arg("fwd"), py::arg("bwd"), py::arg("parts") = 0);
    m.def("forward", [](const CellPtr &c, const Tensor &params, const Tensor &u, const OptTensor &h0, double tol, int64_t max_iter,
                        bool trace, const OptTensor &workspace, const c10::optional<int64_t> &stream, const OptTensor &out) {
        Solve s = unlocked([&] { return solve(*c, params, u, h0, tol, max_iter, trace, workspace, stream, out); });
        return py::make_tuple(s.h, s.iters, object_of(s.trace));
    });
    m.def("backward", [](const CellPtr &c, const Tensor &params, const Tensor &u, const OptTensor &h0, const Tensor &h, const Tensor &g,
                         bool want_dh0, const OptTensor &workspace, const c10::optional<int64_t> &stream, const OptTensor &du,
                         const OptTensor &dparams, const OptTensor &dh0) {
        Grads given;
        if (has(du)) given = {*du, or_none(dparams), or_none(dh0)};
        Grads r = unlocked([&] { return adjoint(*c, params, u, h0, h, g, want_dh0, workspace, stream, has(du) ? &given : nullptr); });
        return py::make_tuple(r.du, r.dparams, object_of(r.dh0));
    });
    m.def("input_projection", [](const Tensor &x, const Tensor &Wx, const OptTensor &bias, int64_t n_heads, const OptTensor &workspace,
                                 const c10::optional<int64_t> &stream, const OptTensor &out) {
        return unlocked([&] { return project(x, Wx, bias, n_heads, workspace, stream, out); });
    });
    m.def("input_projection_backward", [](const Tensor &x, const Tensor &Wx, const Tensor &du, int64_t n_heads, bool want_dx,
                                          bool want_dw, bool want_db, const OptTensor &workspace,
                                          const c10::optional<int64_t> &stream) {
        ProjGrads r = unlocked([&] { return project_backward(x, Wx, du, n_heads, want_dx, want_dw, want_db, workspace, stream); });
        return py::make_tuple(object_of(r.dx), object_of(r.dW), object_of(r.db));
    });
    m.def("release_workspaces", &release_workspaces, py::call_guard<py::gil_scoped_release>());
    m.def("rnn_apply", [](const CellPtr &c, const Tensor &params, const Tensor &u, const OptTensor &h0, double tol, int64_t max_iter) {
        variable_list r = unlocked([&] { return Recurrence::apply(params, u, h0, c, tol, max_iter); });
        return py::make_tuple(r[0], r[1]);
    });
    m.def("input_projection_apply", [](const Tensor &x, const Tensor &Wx, const OptTensor &bias, int64_t n_heads) {
        return unlocked([&] { return Projection::apply(x, Wx, bias, n_heads)[0]; });
    });
    m.def("rnn_layer", [](const CellPtr &c, const Tensor &x, const Tensor &Wx, const OptTensor &bias, const Tensor &params,
                          const OptTensor &h0, int64_t n_heads, double tol, int64_t max_iter) {
        variable_list r = unlocked([&] { return Layer::apply(x, Wx, bias, params, h0, c, n_heads, tol, max_iter); });
        return py::make_tuple(r[0], r[1]);
    });
    m.def("gated_forward", [](const Tensor &u, const OptTensor &h0, const OptTensor &lengths, bool checkpoints, const OptTensor &workspace,
                              const c10::optional<int64_t> &stream, const OptTensor &out, const OptTensor &out_last) {
        GatedOut r = unlocked([&] { return gated_solve(u, h0, lengths, checkpoints, workspace, stream, out, out_last); });
        return py::make_tuple(r.h, r.last, object_of(r.ckpt));
    });
    m.def("gated_backward", [](const Tensor &u, const Tensor &ckpt, const OptTensor &g, const OptTensor &dlast, const OptTensor &lengths,
                               bool want_dh0, const OptTensor &workspace, const c10::optional<int64_t> &stream, const OptTensor &out) {
        GatedGrads r = unlocked([&] { return gated_adjoint(u, ckpt, g, dlast, lengths, want_dh0, workspace, stream, out); });
        return py::make_tuple(r.du, object_of(r.dh0));
    });
    m.def("gated_apply", [](const Tensor &u, const OptTensor &h0, const OptTensor &lengths) {
        variable_list r = unlocked([&] {
            const OptTensor ou(u);
            return Gated::apply(u, h0, lengths, wants_grad({&ou, &h0}));
        });
        return py::make_tuple(r[0], r[1]);
    });
    m.def("gated_layer", [](const Tensor &x, const Tensor &Wx, const OptTensor &bias, const OptTensor &h0, const OptTensor &lengths,
                            int64_t n_heads) {
        variable_list r = unlocked([&] {
            const OptTensor ox(x), ow(Wx);
            return GatedLayer::apply(x, Wx, bias, h0, lengths, n_heads, wants_grad({&ox, &ow, &bias, &h0}));
        });
        return py::make_tuple(r[0], r[1]);
    });
    py::class_<Q4>(m, "ProjectionQ4", "Weights of an input projection in 4 bits, with a bf16 scale for each group of inputs.")
        .def_readonly("packed", &Q4::packed).def_readonly("scales", &Q4::scales)
        .def_readonly("G", &Q4::G).def_readonly("H", &Q4::H).def_readonly("n_heads", &Q4::heads).def_readonly("group", &Q4::group);
    m.def("quantize_projection", [](const Tensor &W, int64_t n_heads, int64_t group, const c10::optional<int64_t> &stream) {
        return unlocked([&] { return q4_quantize(W, n_heads, group, stream); });
    });
    m.def("pack_projection", [](const Tensor &codes, const Tensor &scales, int64_t n_heads, const c10::optional<int64_t> &stream) {
        return unlocked([&] { return q4_pack(codes, scales, n_heads, stream); });
    });
    m.def("dequantize_projection", [](const Q4 &q, const c10::optional<int64_t> &stream) {
        return unlocked([&] { return q4_dequantize(q, stream); });
    });
    m.def("input_projection_q4", [](const Tensor &x, const Q4 &q, const OptTensor &bias, const OptTensor &workspace,
                                    const c10::optional<int64_t> &stream, const OptTensor &out) {
        return unlocked([&] { return q4_project(x, q, bias, workspace, stream, out); });
    });
    m.def("gated_layer_step", [](const Tensor &x, const Q4 &q, const OptTensor &h, const OptTensor &bias, const c10::optional<int64_t> &stream,
                                 const OptTensor &out, const OptTensor &out_h) {
        StepOut r = unlocked([&] { return gated_step(x, q, h, bias, stream, out, out_h); });
        return py::make_tuple(r.y, r.h);
    });
}
