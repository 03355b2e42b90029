// Host state that the entry points of several translation units share
// (defined in dck_api.cu).
#pragma once

#include "common.cuh"

namespace dck {

// Device address of the current device's error word and its SM count (either
// may be null); false if the device cannot be queried.
bool device_state(int** err, int* sms);

// A launch record with the calling thread's timing events (dck_set_timing_events).
LaunchHook thread_hook();

// What dck_last_launch_count reports to the calling thread.
void set_last_launches(int n);

}  // namespace dck
