// Host helpers of the calls around the paged caches.
#pragma once

#include "novakv_internal.cuh"

// Makes the context's device current for the length of a call and puts the caller's back.
struct novakv_device_guard {
    int before = -1;
    bool ok = false;
    explicit novakv_device_guard(const novakv_ctx* ctx) {
        if (cudaGetDevice(&before) != cudaSuccess) return;
        if (before == ctx->cfg.device) before = -1;
        else if (cudaSetDevice(ctx->cfg.device) != cudaSuccess) { before = -1; return; }
        ok = true;
    }
    ~novakv_device_guard() {
        if (before >= 0) cudaSetDevice(before);
    }
    novakv_device_guard(const novakv_device_guard&) = delete;
    novakv_device_guard& operator=(const novakv_device_guard&) = delete;
};
