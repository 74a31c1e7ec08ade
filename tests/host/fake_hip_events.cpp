// The HIP runtime that runs nothing (fake_hip.cpp), writing down as well when an event is recorded.
#define hipEventRecord plain_event_record
#include "fake_hip.cpp"
#undef hipEventRecord

extern "C" int hipEventRecord(void* event, void* stream) {
    calls.push_back("record");
    return plain_event_record(event, stream);
}
