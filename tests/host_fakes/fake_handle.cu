// A scheduler handle with nothing in it, for the calls that only look at its sizes and write its message.
#include "slaq_internal.cuh"

extern "C" slaq_handle* fake_handle(int32_t max_jobs) {
    slaq_handle* const h = new slaq_handle();
    h->max_jobs = max_jobs;
    return h;
}
extern "C" void fake_handle_end(slaq_handle* h) { delete h; }
