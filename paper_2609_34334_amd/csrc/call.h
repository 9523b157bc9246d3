// What an operator's entry point (shard_ops.cpp) needs of the executor in
// api.cpp: this device's state and lock, the configuration, the calling
// thread's error string and statistics, and the timing of its launches.
#pragma once

#include <hip/hip_runtime_api.h>

#include <chrono>
#include <memory>

#include "../../include/hoccl.h"

namespace hoccl {

// Formats the calling thread's error string.
void format_error(const char *fmt, ...) __attribute__((format(printf, 1, 2)));

// One operator call, from open() to done().  The device's lock is held from
// open() until the object goes.
class OpCall {
public:
    OpCall();
    ~OpCall();
    OpCall(const OpCall &) = delete;
    OpCall &operator=(const OpCall &) = delete;

    // Initialises the library on the current device where that is allowed
    // (not while `s` captures), takes the lock and clears the statistics.
    hoccl_status_t open(hipStream_t s);
    int cus() const;
    // The workgroups to launch where `want` would be the automatic choice:
    // at most workgroups_per_step, where that is set, and what a launch takes.
    int budget(unsigned long long want) const;
    // f() enqueues one kernel on the stream and returns its hipError_t.
    template <typename F>
    hoccl_status_t launch(int wg, F &&f) {
        const hoccl_status_t st = before();
        return st != HOCCL_OK ? st : after(wg, f());
    }
    // Fills the statistics.
    void done(unsigned long long hbm_bytes);

private:
    hoccl_status_t before();
    hoccl_status_t after(int wg, hipError_t e);
    struct Impl;
    std::unique_ptr<Impl> impl_;
};

}  // namespace hoccl
